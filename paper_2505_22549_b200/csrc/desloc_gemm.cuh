// Matrix products of many workers' matrices in one launch, on the tensor cores (tcgen05, accumulators in TMEM), with the element-wise work that
// follows each product done on its tiles as they leave TMEM.
//
// C = A B^T per group of matrices, A [m, k], B [n, k] of 16-bit values, sums in fp32.  Either operand lies k-major (rows of k) or m/n-major
// (rows of m or n, a k each): the copies bring 128-byte swizzled boxes of either kind, and the matrix instruction takes both, so nothing is
// ever transposed in memory.  What lies outside a matrix is zeros, filled in by the copy engine.
//
// One block per SM, persistent: a warp requests boxes (TMA) into a ring of stages, a thread issues the products, sixteen warps empty one of two
// accumulators while the other is being filled, and fetch what they need from memory a piece ahead.
//
// Blocks work alone (128 rows of C a tile) or in pairs (256 rows; each brings its own 128 rows of A and half of B, and the tensor cores of both read both
// halves).  What bounds the products of a block alone is its shared memory: for 64 k of a 128 x 256 tile 48 KB are written and read again, 768 cycles of 128 bytes, for
// 512 cycles of products; of a pair each block moves 32 KB in those 512.  What a pair takes is 780 cycles with operands from L2 and nothing else, 570 without bringing any, 900 with
// results that go to memory: 4 x 2048 x 16384 x 2048 with three results 440 us, 1.25 PFLOP/s, in short runs; 4 x 2048 x 2048 x 8192 216 us, 1.27 (cuBLAS sustained: 415 and 220).
#pragma once
#include <atomic>

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "desloc_internal.cuh"
#include "desloc_ops.cuh"

namespace desloc {

constexpr int GEMM_BM = 128, GEMM_BK = 64, GEMM_MAX_STAGES = 16, GEMM_EPI_WARPS = 16, GEMM_THREADS = 128 + 32 * GEMM_EPI_WARPS;
constexpr int GEMM_A_BYTES = GEMM_BM * GEMM_BK * 2;
constexpr int GEMM_SMEM = 227 * 1024 - 2048, GEMM_MAX_GROUPS = 48, GEMM_MAX_MAPS = 64, GEMM_DRAIN_LIMIT = 1 << 22;

// A number of matrices of the same sizes, or a worker's.
struct GemmGroup {
    int tile0;               // number of its first tile in the launch
    int mt, nt, per;         // tiles along m and n, tiles of one matrix
    int m, n, k;
    short a_map, b_map;      // the operands' boxes: of segment s and (dual) half h, the next ones
    short a_mn, b_mn;        // whether the operands lie m- and n-major
    int a_rows;              // rows of A's boxes (k-major): what m leaves of 128; the products read what lies behind them, and nobody reads what comes of that
    int a_batch, b_batch;    // of its first matrix in those maps
    // what the epilogue reads and writes, and how far it is to the next matrix's (elements)
    void *out[3];
    const void *in[2];
    long long out_ld, in_ld, out_batch, in_batch;
    float alpha;
    int first;               // number of its first matrix in a table of the epilogue's
    int wide;                // bits: out (1) and in (2) rows can be moved 16 bytes at a time
    short in_map, out_map;   // boxes of 32 x 32 of what the epilogue reads and writes (out_map + k of out[k]), where the copy engine moves them; else -1
    int io_batch;            // of its first matrix in those maps
    int rotate;              // every tile begins with another k
};

template <typename E>
struct GemmArgs {
    CUtensorMap maps[GEMM_MAX_MAPS];
    GemmGroup groups[GEMM_MAX_GROUPS];
    int ngroups, tiles;
    int tile_n, stages, segments;   // columns of a tile; stages of the ring; pairs of operands that one accumulator sums
    int a_bytes;             // room for A in a stage: of its boxes (the products read 128 rows; what lies behind is never looked at)
    int pairs;               // blocks work in pairs
    int dual;                // the tile's columns are two halves, of two B operands
    int symmetric;           // only tiles that reach the lower triangle, of a product of one operand with itself
    int row_first, row_rest, row_more, row_rest_more;   // of those: tiles in the first row of tiles and in each further one, by division with rest
    uint32_t idesc;          // without the operands' layouts
    int *err;
    int wait_limit;
    E epi;
};

// ---- the machine's instructions ----------------------------------------------------------------------
// (of a pair: the bytes are counted on the first block's barrier)
template <int CG>
__device__ __forceinline__ void tma_load(void *dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar) {
    if constexpr (CG == 1)
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                     :: "r"(smem_u32(dst)), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                     :: "r"(smem_u32(dst)), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
// A box out of shared memory, told to the issuing thread's bulk groups.
__device__ __forceinline__ void tma_store(const CUtensorMap *map, int x, int y, int z, const void *src) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];"
                 :: "l"(map), "r"(x), "r"(y), "r"(z), "r"(smem_u32(src)) : "memory");
}
__device__ __forceinline__ void stores_asked() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
__device__ __forceinline__ void stores_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void stores_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
// The address of the first block's copy of a barrier.
template <int CG>
__device__ __forceinline__ uint32_t first_blocks(const uint64_t *bar) {
    uint32_t at = smem_u32(bar);
    if constexpr (CG == 2) asm volatile("mapa.shared::cluster.u32 %0, %0, 0;" : "+r"(at));
    return at;
}
// Descriptor of an operand's tile in shared memory: 128-byte swizzle; k-major: groups of eight rows 1024 bytes apart; m/n-major: blocks of 64
// columns 8192 bytes apart, groups of eight k 1024 bytes.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr, int mn) {
    return static_cast<uint64_t>((addr >> 4) & 0x3fff) | (static_cast<uint64_t>(mn ? 8192 >> 4 : 1) << 16) | (static_cast<uint64_t>(1024 >> 4) << 32) |
           (1ull << 46) | (2ull << 61);
}
template <int CG>
__device__ __forceinline__ void mma_f16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
    if constexpr (CG == 1)
        asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
                     :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(static_cast<uint32_t>(add)) : "memory");
    else
        asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}"
                     :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(static_cast<uint32_t>(add)) : "memory");
}
// The products so far, done: told to this barrier, of both blocks of a pair.
template <int CG>
__device__ __forceinline__ void mma_commit(uint64_t *bar) {
    if constexpr (CG == 1)
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(smem_u32(bar)) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     :: "r"(smem_u32(bar)), "h"(static_cast<uint16_t>(3)) : "memory");
}
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void bar_init(uint64_t *bar, int count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(smem_u32(bar)), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_expect(uint64_t *bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" :: "r"(smem_u32(bar)), "r"(bytes) : "memory");
}
// A whole warp's wait, with one answer: lanes poll on their own, and at the limit some may have seen what others have not.
__device__ __forceinline__ bool warp_wait(uint64_t *bar, uint32_t parity, int limit) { return __any_sync(0xffffffffu, bar_wait(bar, parity, limit)); }
// One lane of a warp.  (By this instruction the compiler knows that what follows runs in one lane alone and holds addresses and descriptors in uniform registers; behind
// `lane == 0` it did not, and every product took 150 cycles to issue.)
__device__ __forceinline__ bool elect_one() {
    uint32_t one;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(one));
    return one != 0;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// 16 columns of this warp's 32 rows: a row per lane.
__device__ __forceinline__ void tmem_load16(uint32_t addr, float (&v)[16]) {
    uint32_t *r = reinterpret_cast<uint32_t *>(v);
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
                   "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(addr));
}
__device__ __forceinline__ void tmem_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// ---- a warp's 32 x 32 pieces between rows in lanes and rows in memory --------------------------------
// Staged so that global memory sees whole runs of a row: 16-bit values 64 bytes (four lanes), fp32 values 128 bytes (eight lanes).  16-byte pieces change
// places by their row, so that neither side meets bank conflicts.  Rows in lanes are taken 16 columns at a time, half 0 and half 1: sixteen warps, which it takes to hide the
// latencies of all this, leave 96 registers a thread.
struct Piece {
    int rows, cols;   // how much of it lies inside
    bool wide;        // rows begin on 16-byte boundaries
    __device__ __forceinline__ bool none() const { return rows <= 0 || cols <= 0; }
    __device__ __forceinline__ bool whole() const { return wide && rows == 32 && cols == 32; }
};
__device__ __forceinline__ Piece piece_at(const GemmGroup &g, int row0, int col0, bool wide) { return {min(32, g.m - row0), min(32, g.n - col0), wide}; }

// The lane's 16 bytes of row 8 i + lane / 4 (16 bits) or 4 i + lane / 8 (fp32), where they are staged.
__device__ __forceinline__ int spot16(int lane, int i) { return (8 * i + (lane >> 2)) * 64 + (((lane & 3) ^ ((lane >> 3) & 3)) << 4); }
__device__ __forceinline__ int spot32(int lane, int i) { return (4 * i + (lane >> 3)) * 128 + (((lane & 7) ^ ((4 * i + (lane >> 3)) & 7)) << 4); }
// Bytes [16 c, 16 c + 16) of the lane's own row.
__device__ __forceinline__ int place16(int lane, int c) { return lane * 64 + ((c ^ ((lane >> 1) & 3)) << 4); }
__device__ __forceinline__ int place32(int lane, int c) { return lane * 128 + ((c ^ (lane & 7)) << 4); }

// memory -> registers, as it lies there (16 bits: rows on 16-byte boundaries alone)
__device__ __forceinline__ void fetch16(const void *from, long long ld, const Piece &p, int lane, uint4 (&v)[4]) {
    const unsigned short *src = static_cast<const unsigned short *>(from) + (lane >> 2) * ld + 8 * (lane & 3);
    if (p.whole()) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const uint4 *>(src + 8 * i * ld);
        return;
    }
    const int left = p.cols - 8 * (lane & 3);
    if (!p.wide || left <= 0) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (8 * i + (lane >> 2) >= p.rows) continue;
        if (left >= 8) {
            v[i] = *reinterpret_cast<const uint4 *>(src + 8 * i * ld);
        } else {
            uint32_t h[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) h[e] = e < left ? src[8 * i * ld + e] : 0;
            v[i] = make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
        }
    }
}
__device__ __forceinline__ void fetch32(const float *from, long long ld, const Piece &p, int lane, uint4 (&v)[8]) {
    const float *src = from + (lane >> 3) * ld + 4 * (lane & 7);
    if (p.whole()) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = *reinterpret_cast<const uint4 *>(src + 4 * i * ld);
        return;
    }
    const int left = p.cols - 4 * (lane & 7);
    if (left <= 0) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (4 * i + (lane >> 3) >= p.rows) continue;
        if (p.wide && left >= 4) {
            v[i] = *reinterpret_cast<const uint4 *>(src + 4 * i * ld);
        } else {
            uint32_t h[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) h[e] = e < left ? __float_as_uint(src[4 * i * ld + e]) : 0;
            v[i] = make_uint4(h[0], h[1], h[2], h[3]);
        }
    }
}
// registers -> staging area, whence each lane reads its row (behind a __syncwarp()); 16-bit rows on other boundaries come only now, 16 of them at a time.
__device__ __forceinline__ void settle16(char *st, int lane, const void *from, long long ld, const Piece &p, const uint4 (&v)[4]) {
    if (p.wide) {
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4 *>(st + spot16(lane, i)) = v[i];
    } else if (lane < p.cols) {
        const unsigned short *src = static_cast<const unsigned short *>(from) + lane;
        for (int r0 = 0; r0 < p.rows; r0 += 16, src += 16 * ld) {
            unsigned short x[16];
#pragma unroll
            for (int r = 0; r < 16; ++r) x[r] = r0 + r < p.rows ? src[r * ld] : 0;
#pragma unroll
            for (int r = 0; r < 16; ++r) *reinterpret_cast<unsigned short *>(st + place16(r0 + r, lane >> 3) + (lane & 7) * 2) = x[r];
        }
    }
}
__device__ __forceinline__ void settle32(char *st, int lane, const uint4 (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) *reinterpret_cast<uint4 *>(st + spot32(lane, i)) = v[i];
}
__device__ __forceinline__ void row16(const char *st, int lane, int half, uint32_t (&w)[8]) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const uint4 v = *reinterpret_cast<const uint4 *>(st + place16(lane, 2 * half + c));
        w[4 * c] = v.x, w[4 * c + 1] = v.y, w[4 * c + 2] = v.z, w[4 * c + 3] = v.w;
    }
}
__device__ __forceinline__ void row32(const char *st, int lane, int half, float (&v)[16]) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const float4 x = *reinterpret_cast<const float4 *>(st + place32(lane, 4 * half + c));
        v[4 * c] = x.x, v[4 * c + 1] = x.y, v[4 * c + 2] = x.z, v[4 * c + 3] = x.w;
    }
}
// rows in lanes -> staging area (a lane may put where it has read)
__device__ __forceinline__ void put16(char *st, int lane, int half, const uint32_t (&w)[8]) {
#pragma unroll
    for (int c = 0; c < 2; ++c)
        *reinterpret_cast<uint4 *>(st + place16(lane, 2 * half + c)) = make_uint4(w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]);
}
__device__ __forceinline__ void put32(char *st, int lane, int half, const float (&v)[16]) {
#pragma unroll
    for (int c = 0; c < 4; ++c)
        *reinterpret_cast<float4 *>(st + place32(lane, 4 * half + c)) = make_float4(v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3]);
}
// staging area -> memory (behind a __syncwarp()); rows on other than 16-byte boundaries one by one, a column per lane
__device__ __forceinline__ void send16(const char *st, int lane, void *to, long long ld, const Piece &p) {
    unsigned short *dst = static_cast<unsigned short *>(to) + (lane >> 2) * ld + 8 * (lane & 3);
    if (p.whole()) {
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4 *>(dst + 8 * i * ld) = *reinterpret_cast<const uint4 *>(st + spot16(lane, i));
        return;
    }
    if (!p.wide) {
        dst = static_cast<unsigned short *>(to) + lane;
        if (lane < p.cols) {
#pragma unroll 8
            for (int r = 0; r < p.rows; ++r) dst[r * ld] = *reinterpret_cast<const unsigned short *>(st + place16(r, lane >> 3) + (lane & 7) * 2);
        }
        return;
    }
    const int left = p.cols - 8 * (lane & 3);
    if (left <= 0) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (8 * i + (lane >> 2) >= p.rows) continue;
        const uint4 v = *reinterpret_cast<const uint4 *>(st + spot16(lane, i));
        if (left >= 8) {
            *reinterpret_cast<uint4 *>(dst + 8 * i * ld) = v;
        } else {
            const uint32_t h[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < left) dst[8 * i * ld + e] = static_cast<unsigned short>(h[e / 2] >> (16 * (e & 1)));
        }
    }
}
__device__ __forceinline__ void send32(const char *st, int lane, float *to, long long ld, const Piece &p) {
    float *dst = to + (lane >> 3) * ld + 4 * (lane & 7);
    if (p.whole()) {
#pragma unroll
        for (int i = 0; i < 8; ++i) *reinterpret_cast<float4 *>(dst + 4 * i * ld) = *reinterpret_cast<const float4 *>(st + spot32(lane, i));
        return;
    }
    if (!p.wide) {
        if (lane < p.cols) {
#pragma unroll 8
            for (int r = 0; r < p.rows; ++r) to[lane + r * ld] = *reinterpret_cast<const float *>(st + place32(r, lane >> 2) + (lane & 3) * 4);
        }
        return;
    }
    const int left = p.cols - 4 * (lane & 7);
    if (left <= 0) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (4 * i + (lane >> 3) >= p.rows) continue;
        const float4 x = *reinterpret_cast<const float4 *>(st + spot32(lane, i));
        if (left >= 4) {
            *reinterpret_cast<float4 *>(dst + 4 * i * ld) = x;
        } else {
            const float h[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < left) dst[4 * i * ld + e] = h[e];
        }
    }
}

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ float2 unpack_f16(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2 *>(&w)); }
__device__ __forceinline__ float2 unpack_bf16(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }

// ---- the kernel --------------------------------------------------------------------------------------
// Where a tile lies; goes on with the tile's number.  Tiles of a matrix are counted along m first (of a symmetric product row by row, each as far as the diagonal), and a step is
// the same every time: divisions where a group begins alone.
struct TileWalk {
    int group = -1;
    int batch, i, j;             // matrix of the group, tile along m and n
    int at, by_batch, by_i, by_j;   // symmetric: number within the matrix; what a step adds
    // Whether a tile's rows are its columns, too: then what is brought for A serves as B.
    template <int CG, typename A>
    __device__ __forceinline__ bool diagonal(const A &a) const { return a.symmetric && i == j && a.tile_n == CG * GEMM_BM; }
    template <int CG, typename A>
    __device__ __forceinline__ const GemmGroup &find(const A &a, int tile) {
        const int step = gridDim.x / CG, was = group;
        group = max(group, 0);
        while (group + 1 < a.ngroups && a.groups[group + 1].tile0 <= tile) ++group;
        const GemmGroup &g = a.groups[group];
        if (a.symmetric) {
            if (group != was) {
                at = tile - g.tile0;
                batch = at / g.per, by_batch = step / g.per;
                at -= batch * g.per, by_i = step - by_batch * g.per;
            } else {
                batch += by_batch, at += by_i;
                if (at >= g.per) at -= g.per, ++batch;
            }
            // rows of the tiles: row i has 1 + (its last row / tile_n) of them
            int t = at, here = a.row_first, rest = a.row_rest;
            for (i = 0;; ++i) {
                const int some = min(here, g.nt);
                if (t < some) break;
                t -= some;
                here += a.row_more, rest += a.row_rest_more;
                if (rest >= a.tile_n) rest -= a.tile_n, ++here;
            }
            j = t;
        } else if (group != was) {
            const int t = tile - g.tile0, column = t / g.mt;
            i = t - column * g.mt;
            batch = column / g.nt, j = column - batch * g.nt;
            const int columns = step / g.mt;
            by_i = step - columns * g.mt;
            by_batch = columns / g.nt, by_j = columns - by_batch * g.nt;
        } else {
            i += by_i, j += by_j, batch += by_batch;
            if (i >= g.mt) i -= g.mt, ++j;
            if (j >= g.nt) j -= g.nt, ++batch;
        }
        return g;
    }
};

// E, the epilogue, takes 32 x 32 pieces, those that E::wants(group, row, column) says.  What it reads comes one piece ahead: E::READS_BOXES, as a box by the copy engine, pieces in turn
// into the first and second 2 KB of the warp's staging area (of E::STAGING bytes); else as E::Ahead by E::fetch(args, group, batch, row, column, lane, ahead), which
// E::settle(args, group, batch, row, column, staging, lane, ahead) puts there.  E::drain(args, group, batch, row, column, accumulator, staging, input, lane) takes it and the sums, and leaves what is
// written: by E::send(args, group, batch, row, column, staging, lane), or (E::WRITES_BOXES, where the group has maps for it) by E::send_boxes(args, group, batch, row, column, staging, input),
// which one lane calls.  What moves so costs a warp no time: reading, staging and writing 16 bytes a lane were two thirds of what emptying a piece took.
template <typename E, int CG>
__global__ void __launch_bounds__(GEMM_THREADS, 1) gemm_kernel(const __grid_constant__ GemmArgs<E> a) {
    extern __shared__ __align__(1024) char gemm_smem[];
    __shared__ __align__(8) uint64_t full[GEMM_MAX_STAGES], empty[GEMM_MAX_STAGES], ready[2], taken[2], drained, arrived[2 * GEMM_EPI_WARPS];
    __shared__ uint32_t tmem_at, bytes_of[GEMM_MAX_STAGES];
    __shared__ int requested, failed;
    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    uint32_t rank = 0;
    if constexpr (CG == 2) asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    const uint32_t pad = (1024 - (smem_u32(gemm_smem) & 1023)) & 1023;
    char *const ring = gemm_smem + pad;
    const int own_n = a.tile_n / CG, stage_bytes = a.a_bytes + (own_n + 63) / 64 * 64 * (GEMM_BK * 2);
    const int tile0 = blockIdx.x / CG, tile_step = gridDim.x / CG;
    if (threadIdx.x == 0) {
        requested = failed = 0;
        for (int s = 0; s < a.stages; ++s) bar_init(&full[s], 1), bar_init(&empty[s], 1);
        for (int b = 0; b < 2; ++b) bar_init(&ready[b], 1), bar_init(&taken[b], CG * GEMM_EPI_WARPS);
        bar_init(&drained, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0 && elect_one() && tile0 < a.tiles) {   // the descriptions of the first boxes come while earlier kernels end
        TileWalk at;
        const GemmGroup &g = at.find<CG>(a, tile0);
        const auto soon = [&](int map) {
            if (map >= 0) asm volatile("prefetch.tensormap [%0];" :: "l"(&a.maps[map]) : "memory");
        };
        soon(g.a_map), soon(g.b_map);
        if (a.dual || a.segments > 1) soon(g.b_map + 1);
        if (E::READS_BOXES) soon(g.in_map);
        if (E::WRITES_BOXES) soon(g.out_map);
    }
    __syncwarp();
    if (E::READS_BOXES && warp == 3) {
        bar_init(&arrived[lane], 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    static_assert(2 * GEMM_EPI_WARPS == 32, "a barrier for each lane to initialise");
    if (warp == 2) {
        if constexpr (CG == 1) {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" :: "r"(smem_u32(&tmem_at)) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" :: "r"(smem_u32(&tmem_at)) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        }
        // (Only now: the next kernel's blocks may take TMEM and wait for this one's end.  Where one of those could come first on an SM that a block of this kernel has begun on, either would
        // wait for the other.)
        begin_and_let_next_begin();
    }
    tmem_fence_before();
    __syncthreads();
    if constexpr (CG == 2) cluster_sync();
    tmem_fence_after();
    const uint32_t tmem = tmem_at;
    const auto give_up = [&] {
        if (a.err) *reinterpret_cast<volatile int *>(a.err) = 1;
        *reinterpret_cast<volatile int *>(&failed) = 1;
    };

    if (warp == 0) {
        if (elect_one()) {
            TileWalk at;
            int s = 0, asked = 0;
            uint32_t phase = 0;
            bool ok = true, first = true;   // (memory is touched by this thread and the warps below; where the first tile lies is looked up before earlier kernels end)
            for (int tile = tile0; ok && tile < a.tiles; tile += tile_step) {
                const GemmGroup &g = at.find<CG>(a, tile);
                if (first) wait_for_earlier_kernels(), first = false;
                const int m0 = (at.i * CG + rank) * GEMM_BM, steps = (g.k + GEMM_BK - 1) / GEMM_BK;
                const int n0 = a.dual ? at.j * (a.tile_n / 2) : at.j * a.tile_n + rank * own_n;
                const int boxes = (own_n + 63) / 64, turned = g.rotate ? static_cast<int>(tile * 29u % steps) : 0;
                const bool once = at.diagonal<CG>(a);
                const uint32_t bytes = ((g.a_mn ? GEMM_BM : g.a_rows) + (once ? 0 : g.b_mn ? 64 * boxes : own_n)) * (GEMM_BK * 2);
                for (int kk = 0; kk < steps * a.segments; ++kk) {
                    ok = bar_wait(&empty[s], phase ^ 1, a.wait_limit);
                    if (!ok) break;
                    int seg = 0, step = kk;
                    if (step >= steps) seg = 1, step -= steps;
                    if (turned > 0) {
                        step += turned;
                        if (step >= steps) step -= steps;
                    }
                    const int k0 = step * GEMM_BK;
                    char *const sa = ring + s * stage_bytes, *const sb = sa + a.a_bytes;
                    const CUtensorMap *const ma = &a.maps[g.a_map + seg], *const mb = &a.maps[g.b_map + seg];
                    const int za = g.a_batch + at.batch, zb = g.b_batch + at.batch;
                    const uint32_t bar = first_blocks<CG>(&full[s]);
                    bytes_of[s] = bytes;
                    if (rank == 0) bar_expect(&full[s], CG * bytes);
                    if (g.a_mn) {
                        for (int x = 0; x < GEMM_BM; x += 64) tma_load<CG>(sa + x * (GEMM_BK * 2), ma, m0 + x, k0, za, bar);
                    } else {
                        tma_load<CG>(sa, ma, k0, m0, za, bar);
                    }
                    if (once) {
                    } else if (g.b_mn) {
                        for (int x = 0; x < boxes; ++x) tma_load<CG>(sb + x * (64 * GEMM_BK * 2), mb, n0 + 64 * x, k0, zb, bar);
                    } else if (!a.dual) {
                        tma_load<CG>(sb, mb, k0, n0, zb, bar);
                    } else if (CG == 2) {   // a half each
                        tma_load<CG>(sb, mb + rank, k0, n0, zb, bar);
                    } else {
                        tma_load<CG>(sb, mb, k0, n0, zb, bar);
                        tma_load<CG>(sb + a.tile_n * GEMM_BK, mb + 1, k0, n0, zb, bar);
                    }
                    ++asked;
                    if (++s == a.stages) s = 0, phase ^= 1;
                }
            }
            requested = asked;
            if (!ok) give_up();
            // the products have read what this block brought (and told so) before it may leave
            for (int x = max(0, asked - a.stages); ok && x < asked; ++x) ok = bar_wait(&empty[x % a.stages], (x / a.stages) & 1, a.wait_limit);
            if (!ok) give_up();
        }
        __syncwarp();
    } else if (warp == 1) {
        if (rank == 0 && elect_one()) {
            TileWalk at;
            int s = 0, buf = 0;
            uint32_t phase = 0, turn = 0;
            bool ok = true;
            wait_for_earlier_kernels();   // (nothing is asked for before: what earlier kernels take is no part of the wait below, whose polls are counted)
            for (int tile = tile0; ok && tile < a.tiles; tile += tile_step) {
                const GemmGroup &g = at.find<CG>(a, tile);
                const int steps = (g.k + GEMM_BK - 1) / GEMM_BK * a.segments;
                ok = bar_wait(&taken[buf], turn ^ 1, a.wait_limit);
                if (!ok) break;
                tmem_fence_after();
                const uint32_t d = tmem + buf * 256, idesc = a.idesc | (g.a_mn ? 1u << 15 : 0) | (g.b_mn ? 1u << 16 : 0);
                const bool once = at.diagonal<CG>(a);
                const uint32_t ka = (g.a_mn ? 2048 : 32) >> 4, kb = (g.b_mn ? 2048 : 32) >> 4;
                for (int kk = 0; kk < steps; ++kk) {
                    ok = bar_wait(&full[s], phase, a.wait_limit);
                    if (!ok) break;
                    tmem_fence_after();
                    const uint32_t sa = smem_u32(ring + s * stage_bytes);
                    const uint64_t da = operand_desc(sa, g.a_mn), db = once ? da : operand_desc(sa + a.a_bytes, g.b_mn);
#pragma unroll
                    for (int x = 0; x < GEMM_BK / 16; ++x) mma_f16<CG>(d, da + x * ka, db + x * kb, idesc, kk > 0 || x > 0);
                    mma_commit<CG>(&empty[s]);
                    if (++s == a.stages) s = 0, phase ^= 1;
                }
                if (!ok) break;
                mma_commit<CG>(&ready[buf]);
                buf ^= 1;
                if (buf == 0) turn ^= 1;
            }
            if (!ok) {   // the products that are on their way end first
                give_up();
                mma_commit<CG>(&drained);
                bar_wait(&drained, 0, GEMM_DRAIN_LIMIT);
            }
        }
        __syncwarp();
    } else if (warp >= 4) {
        constexpr int STEP = GEMM_EPI_WARPS / 4 * 32;   // columns that the warps take at a time
        const int quadrant = warp & 3, c0 = (warp - 4) / 4 * 32;
        char *const st = ring + a.stages * stage_bytes + (warp - 4) * E::STAGING;
        uint64_t *const came = &arrived[2 * (warp - 4)];
        const int out_n = a.dual ? a.tile_n / 2 : a.tile_n;
        const int rows = (rank * 4 + quadrant) * 32;
        TileWalk at;
        typename E::Ahead ahead;
        int buf = 0, tile = tile0, c = c0, asked = 0, taken_boxes = 0;
        uint32_t turn = 0;
        const GemmGroup *g = nullptr;
        // what the next piece reads
        const auto ask = [&] {
            const int row0 = at.i * (CG * GEMM_BM) + rows, col0 = at.j * out_n + c;
            if (c0 >= out_n || !E::wants(*g, row0, col0)) return;
            if constexpr (E::READS_BOXES) {
                if (g->in_map < 0) return;
                if (elect_one()) {
                    uint64_t *const bar = &came[asked & 1];
                    bar_expect(bar, 2048);
                    tma_load<1>(st + (asked & 1) * 2048, &a.maps[g->in_map], col0, row0, g->io_batch + at.batch, smem_u32(bar));
                }
                __syncwarp();
                ++asked;
            } else {
                E::fetch(a, *g, at.batch, row0, col0, lane, ahead);
            }
        };
        if (tile < a.tiles) {
            g = &at.find<CG>(a, tile);
            wait_for_earlier_kernels();
            ask();
        }
        bool ok = true;
        while (tile < a.tiles) {
            if (c == c0) {
                ok = warp_wait(&ready[buf], turn, a.wait_limit);
                if (!ok) break;
                tmem_fence_after();
            }
            const GemmGroup &here = *g;
            const int batch = at.batch, row0 = at.i * (CG * GEMM_BM) + rows, col0 = at.j * out_n + c;
            const uint32_t d = tmem + buf * 256 + c + (static_cast<uint32_t>(32 * quadrant) << 16);
            const bool wanted = c0 < out_n && E::wants(here, row0, col0), reads = E::READS_BOXES && wanted && here.in_map >= 0;
            const char *const input = st + (taken_boxes & 1) * 2048;
            // the piece before has left the staging area
            if constexpr (E::WRITES_BOXES) {
                if (elect_one()) stores_read();
            }
            __syncwarp();
            if constexpr (!E::READS_BOXES) if (wanted) E::settle(a, here, batch, row0, col0, st, lane, ahead);
            c += STEP;
            const bool last = c >= out_n;
            if (last) {
                c = c0, tile += tile_step;
                if (tile < a.tiles) g = &at.find<CG>(a, tile);
            }
            if (tile < a.tiles) ask();
            if (reads) {
                ok = warp_wait(&came[taken_boxes & 1], (taken_boxes >> 1) & 1, a.wait_limit);
                if (!ok) break;
                ++taken_boxes;
            }
            __syncwarp();
            if (wanted) E::drain(a, here, batch, row0, col0, d, st, input, lane);
            if constexpr (E::WRITES_BOXES) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            tmem_fence_before();
            __syncwarp();
            if (last) {
                // (no more than that the accumulator has been read is told: a release to the other block would wait for this warp's stores)
                if (lane == 0) {
                    if constexpr (CG == 1) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" :: "r"(smem_u32(&taken[buf])) : "memory");
                    else asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" :: "r"(first_blocks<CG>(&taken[buf])) : "memory");
                }
                buf ^= 1;
                if (buf == 0) turn ^= 1;
            }
            if (wanted) {
                if constexpr (E::WRITES_BOXES) {
                    if (here.out_map >= 0) {
                        if (elect_one()) {
                            E::send_boxes(a, here, batch, row0, col0, st, input);
                            stores_asked();
                        }
                        continue;
                    }
                }
                E::send(a, here, batch, row0, col0, st, lane);
            }
        }
        if (!ok) give_up();
        // what is on its way lands first
        if constexpr (E::READS_BOXES) {
            for (; taken_boxes < asked; ++taken_boxes) bar_wait(&came[taken_boxes & 1], (taken_boxes >> 1) & 1, GEMM_DRAIN_LIMIT);
        }
        __syncwarp();
        if constexpr (E::WRITES_BOXES) {
            if (elect_one()) stores_done();
        }
        __syncwarp();
    }
    tmem_fence_before();
    __syncthreads();
    int others = 0, fell = failed;
    if constexpr (CG == 2) {
        cluster_sync();
        uint32_t where, flag;
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(where) : "r"(smem_u32(&requested)), "r"(rank ^ 1));
        asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(others) : "r"(where) : "memory");
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(where) : "r"(smem_u32(&failed)), "r"(rank ^ 1));
        asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(flag) : "r"(where) : "memory");
        fell |= static_cast<int>(flag);
    }
    if (fell && rank == 0 && threadIdx.x == 0) {
        // Copies that are on their way land before anyone leaves.  Of a stage that one block of a pair has requested and the other has not, the other's
        // part is made up: asked for less, or told as done.
        const int mine = requested, most = CG == 2 ? max(mine, others) : mine, both = CG == 2 ? min(mine, others) : mine;
        for (int x = max(0, most - a.stages); x < most; ++x) {
            const int s = x % a.stages;
            if (x >= both && mine < most) {
                uint32_t where, bytes;
                asm volatile("mapa.shared::cluster.u32 %0, %1, 1;" : "=r"(where) : "r"(smem_u32(&bytes_of[s])));
                asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(bytes) : "r"(where) : "memory");
                bar_expect(&full[s], bytes);
            }
            if (x >= both && mine == most)
                asm volatile("mbarrier.complete_tx.relaxed.cluster.shared::cluster.b64 [%0], %1;" :: "r"(smem_u32(&full[s])), "r"(bytes_of[s]) : "memory");
            bar_wait(&full[s], (x / a.stages) & 1, GEMM_DRAIN_LIMIT);
        }
    }
    __syncwarp();
    if constexpr (CG == 2) cluster_sync();   // (what one block reads of the other has been read)
    if (warp == 2) {
        tmem_fence_after();
        if constexpr (CG == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" :: "r"(tmem) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" :: "r"(tmem) : "memory");
    }
}

// ---- host --------------------------------------------------------------------------------------------
// Boxes of 64 x `rows` values (k-major: 64 k of so many rows; m/n-major: 64 columns of so many k) of `batch` matrices of `outer` rows of `inner` 16-bit values.
// columns = 32: of 32 columns, swizzled by 64 bytes, as the epilogues stage them.
cudaError_t encode_boxes(CUtensorMap *map, const void *data, bool bf16, int64_t inner, int64_t outer, int64_t batch, int64_t ld, int64_t batch_ld, int rows, int columns = 64);

// Whether rows `ld` elements apart from `data` on can be fetched by the copy engine: 16-byte boundaries.
inline bool boxes_fit(const void *data, int64_t ld) { return ((reinterpret_cast<uintptr_t>(data) | static_cast<uintptr_t>(ld * 2)) & 15u) == 0; }

// Rows of a k-major box of an A with m rows.
inline int box_rows(int64_t m) { return static_cast<int>(std::min<int64_t>(GEMM_BM, (m + 7) / 8 * 8)); }

// How a launch is cut: columns of a tile (dual: of both halves together), and whether blocks work in pairs.
struct GemmCut {
    int tile_n;
    bool pairs;
    int out_n(bool dual) const { return dual ? tile_n / 2 : tile_n; }
    int box_n(bool dual) const { return dual || pairs ? tile_n / 2 : tile_n; }   // rows of a k-major box of B
};
inline int tiles_of(int m, int n, const GemmCut &cut, bool dual, bool symmetric) {
    const int bm = GEMM_BM * (cut.pairs ? 2 : 1), tile_n = cut.out_n(dual);
    const int mt = (m + bm - 1) / bm, nt = (n + tile_n - 1) / tile_n;
    if (!symmetric) return mt * nt;
    int all = 0;
    for (int i = 0; i < mt; ++i) all += std::min((i * bm + bm - 1) / tile_n + 1, nt);
    return all;
}
// How many tiles a launch has, and how many of those lie on the diagonal of a symmetric product and bring one operand.
struct TileCount {
    int64_t all, once;
};
// The cut that is done first: rounds of tiles (half of what the last round leaves empty counted: tiles differ in k), a tile as long as bringing and multiplying 64 k takes, or as
// emptying it (some 1500 cycles for the 128 columns that the warps take at a time); and what a launch takes before and behind.  In cycles for 64 k, from products of 8192 k: 775 for
// 256, 672 for 192 and 657 for 128 columns of a pair, 844, 740 and 615 of a block alone; tiles that bring one operand a quarter less.  Few rows (up to FEW_ROWS): what
// takes time is B from memory, some 6 cycles a column when all SMs read.  tiles(cut): a TileCount, all with k of about `k`.
constexpr int64_t FEW_ROWS = 64;
template <typename F>
GemmCut pick_cut(bool dual, int64_t m, int64_t k, const F &tiles) {
    GemmCut best{};
    int64_t least = 0;
    for (int pairs = m > FEW_ROWS ? 1 : 0; pairs >= 0; --pairs)
        for (int n = 256; n >= (pairs ? 128 : 64); n -= 64) {
            const GemmCut cut{n, pairs != 0};
            const TileCount count = tiles(cut);
            const int64_t slots = pairs ? NUM_SMS / 2 : NUM_SMS, step = m <= FEW_ROWS ? 60 + 6 * n : pairs ? 440 + 13 * n / 10 : 384 + 9 * n / 5;
            const int64_t products = (k + GEMM_BK - 1) / GEMM_BK * (step * (4 * count.all - count.once) / (4 * count.all)), empty = (cut.out_n(dual) + 127) / 128 * 1500;
            const int64_t each = std::max(products, empty) + 200;
            const int64_t cost = (count.all + slots - 1) / slots * each + std::max(count.all, slots) * each / slots + 2 * std::min(products, empty);
            if (!best.tile_n || cost < least) best = cut, least = cost;
        }
    return best;
}

template <typename E>
void begin_gemm(GemmArgs<E> &a, bool bf16, const GemmCut &cut, bool dual, bool symmetric, int segments) {
    a.ngroups = a.tiles = a.a_bytes = 0;
    a.tile_n = cut.tile_n, a.pairs = cut.pairs, a.dual = dual, a.symmetric = symmetric, a.segments = segments;
    const int bm = GEMM_BM * (cut.pairs ? 2 : 1);
    a.row_first = (bm - 1) / cut.tile_n + 1, a.row_rest = (bm - 1) % cut.tile_n;
    a.row_more = bm / cut.tile_n, a.row_rest_more = bm % cut.tile_n;
    const uint32_t type = bf16 ? 1 : 0;
    a.idesc = 1u << 4 | type << 7 | type << 10 | static_cast<uint32_t>(cut.tile_n >> 3) << 17 | static_cast<uint32_t>((cut.pairs ? 2 : 1) * GEMM_BM >> 4) << 24;
}
// The next group, of `count` matrices: its sizes and tiles; the rest is the caller's.
template <typename E>
GemmGroup &add_group(GemmArgs<E> &a, int m, int n, int k, int count) {
    GemmGroup &g = a.groups[a.ngroups++];
    g = GemmGroup{};
    const GemmCut cut{a.tile_n, a.pairs != 0};
    const int out_n = cut.out_n(a.dual), bm = GEMM_BM * (a.pairs ? 2 : 1);
    g.tile0 = a.tiles;
    g.m = m, g.n = n, g.k = k, g.a_rows = box_rows(m);
    g.in_map = g.out_map = -1;
    g.mt = (m + bm - 1) / bm, g.nt = (n + out_n - 1) / out_n;
    g.per = tiles_of(m, n, cut, a.dual, a.symmetric);
    a.tiles += g.per * count;
    // Few rows: all that is read is B, once, and all blocks at once would read the same columns of rows that lie a power of two apart, of which a few of the memory's channels
    // have to bring all (the 8192 columns of down, one row of h: 1.7 TB/s).
    g.rotate = m <= FEW_ROWS;
    return g;
}

// Raises a kernel's limit of shared memory, once on each device.
template <typename E, int CG>
cudaError_t gemm_ready() {
    static std::atomic<uint64_t> done{0};
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess || (device < 64 && (done.load() >> device & 1))) return e;
    e = cudaFuncSetAttribute(gemm_kernel<E, CG>, cudaFuncAttributeMaxDynamicSharedMemorySize, GEMM_SMEM);
    if (e == cudaSuccess && device < 64) done.fetch_or(1ull << device);
    return e;
}

template <typename E, int CG>
cudaError_t launch_gemm(GemmArgs<E> &a, cudaStream_t stream) {
    const cudaError_t e = gemm_ready<E, CG>();
    if (e != cudaSuccess) return e;
    for (int i = 0; i < a.ngroups; ++i) a.a_bytes = std::max(a.a_bytes, (a.groups[i].a_mn ? GEMM_BM : a.groups[i].a_rows) * GEMM_BK * 2);
    const int stage = a.a_bytes + (a.tile_n / CG + 63) / 64 * 64 * GEMM_BK * 2;
    // (behind the last stage there is room for the rows of A that it lacks)
    a.stages = std::min(GEMM_MAX_STAGES, (GEMM_SMEM - 1024 - std::max(GEMM_EPI_WARPS * E::STAGING, GEMM_A_BYTES)) / stage);
    cudaLaunchConfig_t lc{};
    lc.gridDim = dim3(static_cast<unsigned>(CG * std::min(a.tiles, NUM_SMS / CG)));
    lc.blockDim = dim3(GEMM_THREADS);
    lc.dynamicSmemBytes = 1024 + static_cast<size_t>(a.stages) * stage + std::max(GEMM_EPI_WARPS * E::STAGING, GEMM_A_BYTES);
    lc.stream = stream;
    cudaLaunchAttribute at[2]{};
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = CG, at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    lc.attrs = at;
    lc.numAttrs = CG == 2 ? 2 : 1;
    void *args[1] = {&a};
    return cudaLaunchKernelExC(&lc, reinterpret_cast<const void *>(gemm_kernel<E, CG>), args);
}
template <typename E>
cudaError_t launch_gemm(GemmArgs<E> &a, int *err, int wait_limit, cudaStream_t stream, int *launches) {
    if (a.tiles == 0) return cudaSuccess;
    a.err = err, a.wait_limit = wait_limit;
    const cudaError_t e = a.pairs ? launch_gemm<E, 2>(a, stream) : launch_gemm<E, 1>(a, stream);
    if (e == cudaSuccess) ++*launches;
    return e;
}

}  // namespace desloc
