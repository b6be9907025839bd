// Matrix products of many workers' matrices in one launch, on the tensor cores (tcgen05, accumulators in TMEM), with the element-wise work that
// follows each product done on its tiles as they leave TMEM.
//
// C = A B^T per group of matrices, A [m, k], B [n, k] of 16-bit values, sums in fp32.  Either operand lies k-major (rows of k) or m/n-major
// (rows of m or n, a k each): the copies bring 128-byte swizzled boxes of either kind, and the matrix instruction takes both, so nothing is
// ever transposed in memory.  What lies outside a matrix is zeros, filled in by the copy engine.
//
// One block per SM, persistent: a warp requests boxes (TMA) into a ring of stages, a thread issues the products, eight warps empty one of two
// accumulators while the other is being filled.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "desloc_internal.cuh"
#include "desloc_ops.cuh"

namespace desloc {

constexpr int GEMM_BM = 128, GEMM_BK = 64, GEMM_MAX_STAGES = 8, GEMM_EPI_WARPS = 8, GEMM_THREADS = 128 + 32 * GEMM_EPI_WARPS;
constexpr int GEMM_A_BYTES = GEMM_BM * GEMM_BK * 2, GEMM_STAGING = 4096;   // staging: of every warp that empties accumulators
constexpr int GEMM_SMEM = 227 * 1024 - 2048, GEMM_MAX_GROUPS = 48, GEMM_MAX_MAPS = 64, GEMM_DRAIN_LIMIT = 1 << 22;

// A number of matrices of the same sizes, or a worker's.
struct GemmGroup {
    int tile0;               // number of its first tile in the launch
    int mt, nt, per;         // tiles along m and n, tiles of one matrix
    int m, n, k;
    short a_map, b_map;      // the operands' boxes: of segment s and (dual) half h, the next ones
    short a_mn, b_mn;        // whether the operands lie m- and n-major
    int a_batch, b_batch;    // of its first matrix in those maps
    // what the epilogue reads and writes, and how far it is to the next matrix's (elements)
    void *out[3];
    const void *in[2];
    long long out_ld, in_ld, out_batch, in_batch;
    float alpha;
    int first;               // number of its first matrix in a table of the epilogue's
    int wide;                // bits: out (1) and in (2) rows can be moved 16 bytes at a time
};

template <typename E>
struct GemmArgs {
    CUtensorMap maps[GEMM_MAX_MAPS];
    GemmGroup groups[GEMM_MAX_GROUPS];
    int ngroups, tiles;
    int tile_n, stages, segments;   // columns of a tile; stages of the ring; pairs of operands that one accumulator sums
    int dual;                // the tile's columns are two halves, of two B operands
    int symmetric;           // only tiles that reach the lower triangle
    uint32_t idesc;          // without the operands' layouts
    int *err;
    int wait_limit;
    E epi;
};

// ---- the machine's instructions ----------------------------------------------------------------------
__device__ __forceinline__ void tma_load(void *dst, const CUtensorMap *map, int x, int y, int z, uint64_t *bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 :: "r"(smem_u32(dst)), "l"(map), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar)) : "memory");
}
// Descriptor of an operand's tile in shared memory: 128-byte swizzle; k-major: groups of eight rows 1024 bytes apart; m/n-major: blocks of 64
// columns 8192 bytes apart, groups of eight k 1024 bytes.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr, int mn) {
    return static_cast<uint64_t>((addr >> 4) & 0x3fff) | (static_cast<uint64_t>(mn ? 8192 >> 4 : 1) << 16) | (static_cast<uint64_t>(1024 >> 4) << 32) |
           (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ void mma_f16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
                 :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(static_cast<uint32_t>(add)) : "memory");
}
__device__ __forceinline__ void mma_commit(uint64_t *bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void bar_init(uint64_t *bar, int count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(smem_u32(bar)), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_expect(uint64_t *bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" :: "r"(smem_u32(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint64_t *bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" :: "r"(smem_u32(bar)) : "memory");
}
// 32 columns of this warp's 32 rows: a row per lane.
__device__ __forceinline__ void tmem_load32(uint32_t addr, float (&v)[32]) {
    uint32_t *r = reinterpret_cast<uint32_t *>(v);
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,"
                 "%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
                   "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
                   "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
                   "=r"(r[31])
                 : "r"(addr));
}
__device__ __forceinline__ void tmem_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// ---- a warp's 32 x 32 pieces between rows in lanes and rows in memory --------------------------------
// Staged so that global memory sees whole runs of a row: 16-bit values 64 bytes (four lanes), fp32 values 128 bytes (eight lanes).  16-byte pieces change
// places by their row, so that neither side meets bank conflicts.
struct Piece {
    int rows, cols;   // how much of it lies inside
    bool wide;        // rows begin on 16-byte boundaries
};

template <typename F>
__device__ __forceinline__ void visit16(const Piece &p, int lane, const F &f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = 8 * i + (lane >> 2), c = lane & 3;
        if (row < p.rows && 8 * c < p.cols) f(row, 8 * c, row * 64 + ((c ^ ((row >> 1) & 3)) << 4));
    }
}
__device__ __forceinline__ int place16(int lane, int c) { return lane * 64 + ((c ^ ((lane >> 1) & 3)) << 4); }

// memory -> w: 16 words of two values, the lane's row
__device__ __forceinline__ void load_piece16(char *st, int lane, const void *from, long long ld, const Piece &p, uint32_t (&w)[16]) {
    const unsigned short *src = static_cast<const unsigned short *>(from);
    __syncwarp();
    visit16(p, lane, [&](int row, int col, int at) {
        uint4 v;
        if (p.wide && col + 8 <= p.cols) {
            v = *reinterpret_cast<const uint4 *>(src + row * ld + col);
        } else {
            uint32_t h[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) h[e] = col + e < p.cols ? src[row * ld + col + e] : 0;
            v = make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
        }
        *reinterpret_cast<uint4 *>(st + at) = v;
    });
    __syncwarp();
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const uint4 v = *reinterpret_cast<const uint4 *>(st + place16(lane, c));
        w[4 * c] = v.x, w[4 * c + 1] = v.y, w[4 * c + 2] = v.z, w[4 * c + 3] = v.w;
    }
}
__device__ __forceinline__ void store_piece16(char *st, int lane, void *to, long long ld, const Piece &p, const uint32_t (&w)[16]) {
    unsigned short *dst = static_cast<unsigned short *>(to);
    __syncwarp();
#pragma unroll
    for (int c = 0; c < 4; ++c) *reinterpret_cast<uint4 *>(st + place16(lane, c)) = make_uint4(w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]);
    __syncwarp();
    visit16(p, lane, [&](int row, int col, int at) {
        const uint4 v = *reinterpret_cast<const uint4 *>(st + at);
        if (p.wide && col + 8 <= p.cols) {
            *reinterpret_cast<uint4 *>(dst + row * ld + col) = v;
        } else {
            const uint32_t h[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (col + e < p.cols) dst[row * ld + col + e] = static_cast<unsigned short>(h[e / 2] >> (16 * (e & 1)));
        }
    });
}

template <typename F>
__device__ __forceinline__ void visit32(const Piece &p, int lane, const F &f) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int row = 4 * i + (lane >> 3), c = lane & 7;
        if (row < p.rows && 4 * c < p.cols) f(row, 4 * c, row * 128 + ((c ^ (row & 7)) << 4));
    }
}
__device__ __forceinline__ int place32(int lane, int c) { return lane * 128 + ((c ^ (lane & 7)) << 4); }

__device__ __forceinline__ void load_piece32(char *st, int lane, const float *src, long long ld, const Piece &p, float (&v)[32]) {
    __syncwarp();
    visit32(p, lane, [&](int row, int col, int at) {
        float4 x;
        if (p.wide && col + 4 <= p.cols) {
            x = *reinterpret_cast<const float4 *>(src + row * ld + col);
        } else {
            float h[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) h[e] = col + e < p.cols ? src[row * ld + col + e] : 0.f;
            x = make_float4(h[0], h[1], h[2], h[3]);
        }
        *reinterpret_cast<float4 *>(st + at) = x;
    });
    __syncwarp();
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        const float4 x = *reinterpret_cast<const float4 *>(st + place32(lane, c));
        v[4 * c] = x.x, v[4 * c + 1] = x.y, v[4 * c + 2] = x.z, v[4 * c + 3] = x.w;
    }
}
__device__ __forceinline__ void store_piece32(char *st, int lane, float *dst, long long ld, const Piece &p, const float (&v)[32]) {
    __syncwarp();
#pragma unroll
    for (int c = 0; c < 8; ++c) *reinterpret_cast<float4 *>(st + place32(lane, c)) = make_float4(v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3]);
    __syncwarp();
    visit32(p, lane, [&](int row, int col, int at) {
        const float4 x = *reinterpret_cast<const float4 *>(st + at);
        if (p.wide && col + 4 <= p.cols) {
            *reinterpret_cast<float4 *>(dst + row * ld + col) = x;
        } else {
            const float h[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (col + e < p.cols) dst[row * ld + col + e] = h[e];
        }
    });
}

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ float2 unpack_f16(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2 *>(&w)); }
__device__ __forceinline__ float2 unpack_bf16(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }

// ---- the kernel --------------------------------------------------------------------------------------
// Where a tile lies; advances with the tile's number.
struct TileWalk {
    int group = 0;
    int batch, i, j;   // matrix of the group, tile along m and n
    template <typename A>
    __device__ __forceinline__ const GemmGroup &find(const A &a, int tile) {
        while (group + 1 < a.ngroups && a.groups[group + 1].tile0 <= tile) ++group;
        const GemmGroup &g = a.groups[group];
        int t = tile - g.tile0;
        batch = t / g.per;
        t -= batch * g.per;
        if (a.symmetric) {   // row i of tiles reaches as far as the diagonal
            for (i = 0;; ++i) {
                const int here = min((i * GEMM_BM + GEMM_BM - 1) / a.tile_n + 1, g.nt);
                if (t < here) break;
                t -= here;
            }
            j = t;
        } else {
            j = t / g.mt;
            i = t - j * g.mt;
        }
        return g;
    }
};

// E: the epilogue.  E::piece(args, group, batch, i, j, accumulator, column, staging, quadrant, lane) takes 32 columns (dual: of both halves) of a quadrant of 32 rows.
template <typename E>
__global__ void __launch_bounds__(GEMM_THREADS, 1) gemm_kernel(const __grid_constant__ GemmArgs<E> a) {
    extern __shared__ __align__(1024) char gemm_smem[];
    __shared__ __align__(8) uint64_t full[GEMM_MAX_STAGES], empty[GEMM_MAX_STAGES], ready[2], taken[2], drained;
    __shared__ uint32_t tmem_at;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t pad = (1024 - (smem_u32(gemm_smem) & 1023)) & 1023;
    char *const ring = gemm_smem + pad;
    const int stage_bytes = GEMM_A_BYTES + a.tile_n * (GEMM_BK * 2);
    begin_and_let_next_begin();
    if (threadIdx.x == 0) {
        for (int s = 0; s < a.stages; ++s) bar_init(&full[s], 1), bar_init(&empty[s], 1);
        for (int b = 0; b < 2; ++b) bar_init(&ready[b], 1), bar_init(&taken[b], GEMM_EPI_WARPS);
        bar_init(&drained, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" :: "r"(smem_u32(&tmem_at)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const uint32_t tmem = tmem_at;
    wait_for_earlier_kernels();
    const auto give_up = [&] {
        if (a.err) *reinterpret_cast<volatile int *>(a.err) = 1;
    };

    if (warp == 0) {
        if (lane == 0) {
            TileWalk at;
            int s = 0, asked = 0;
            uint32_t phase = 0;
            bool ok = true;
            for (int tile = blockIdx.x; ok && tile < a.tiles; tile += gridDim.x) {
                const GemmGroup &g = at.find(a, tile);
                const int m0 = at.i * GEMM_BM, n0 = at.j * (a.dual ? a.tile_n / 2 : a.tile_n), steps = (g.k + GEMM_BK - 1) / GEMM_BK;
                for (int kk = 0; ok && kk < steps * a.segments; ++kk) {
                    ok = bar_wait(&empty[s], phase ^ 1, a.wait_limit);
                    if (!ok) break;
                    const int seg = kk >= steps ? 1 : 0, k0 = (kk - seg * steps) * GEMM_BK;
                    char *const sa = ring + s * stage_bytes, *const sb = sa + GEMM_A_BYTES;
                    const CUtensorMap *const ma = &a.maps[g.a_map + seg], *const mb = &a.maps[g.b_map + seg];
                    const int za = g.a_batch + at.batch, zb = g.b_batch + at.batch;
                    bar_expect(&full[s], stage_bytes);
                    if (g.a_mn) {
                        for (int x = 0; x < GEMM_BM; x += 64) tma_load(sa + x * (GEMM_BK * 2), ma, m0 + x, k0, za, &full[s]);
                    } else {
                        tma_load(sa, ma, k0, m0, za, &full[s]);
                    }
                    if (g.b_mn) {
                        for (int x = 0; x < a.tile_n; x += 64) tma_load(sb + x * (GEMM_BK * 2), mb, n0 + x, k0, zb, &full[s]);
                    } else {
                        tma_load(sb, mb, k0, n0, zb, &full[s]);
                        if (a.dual) tma_load(sb + a.tile_n * GEMM_BK, mb + 1, k0, n0, zb, &full[s]);
                    }
                    ++asked;
                    if (++s == a.stages) s = 0, phase ^= 1;
                }
            }
            if (!ok) {   // the copies that are on their way land first
                give_up();
                for (int x = max(0, asked - a.stages); x < asked; ++x) bar_wait(&full[x % a.stages], (x / a.stages) & 1, GEMM_DRAIN_LIMIT);
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0) {
            TileWalk at;
            int s = 0, buf = 0;
            uint32_t phase = 0, turn = 0;
            bool ok = true;
            for (int tile = blockIdx.x; ok && tile < a.tiles; tile += gridDim.x) {
                const GemmGroup &g = at.find(a, tile);
                const int steps = (g.k + GEMM_BK - 1) / GEMM_BK * a.segments;
                ok = bar_wait(&taken[buf], turn ^ 1, a.wait_limit);
                if (!ok) break;
                tmem_fence_after();
                const uint32_t d = tmem + buf * 256, idesc = a.idesc | (g.a_mn ? 1u << 15 : 0) | (g.b_mn ? 1u << 16 : 0);
                const uint32_t ka = (g.a_mn ? 2048 : 32) >> 4, kb = (g.b_mn ? 2048 : 32) >> 4;
                for (int kk = 0; kk < steps; ++kk) {
                    ok = bar_wait(&full[s], phase, a.wait_limit);
                    if (!ok) break;
                    tmem_fence_after();
                    const uint32_t sa = smem_u32(ring + s * stage_bytes);
                    const uint64_t da = operand_desc(sa, g.a_mn), db = operand_desc(sa + GEMM_A_BYTES, g.b_mn);
#pragma unroll
                    for (int x = 0; x < GEMM_BK / 16; ++x) mma_f16(d, da + x * ka, db + x * kb, idesc, kk > 0 || x > 0);
                    mma_commit(&empty[s]);
                    if (++s == a.stages) s = 0, phase ^= 1;
                }
                if (!ok) break;
                mma_commit(&ready[buf]);
                buf ^= 1;
                if (buf == 0) turn ^= 1;
            }
            if (!ok) {   // the products that are on their way end first
                give_up();
                mma_commit(&drained);
                bar_wait(&drained, 0, GEMM_DRAIN_LIMIT);
            }
        }
        __syncwarp();
    } else if (warp >= 4) {
        const int quadrant = warp & 3, half = (warp - 4) >> 2;
        char *const st = ring + a.stages * stage_bytes + (warp - 4) * GEMM_STAGING;
        TileWalk at;
        int buf = 0;
        uint32_t turn = 0;
        const int out_n = a.dual ? a.tile_n / 2 : a.tile_n;
        for (int tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
            const GemmGroup &g = at.find(a, tile);
            if (!bar_wait(&ready[buf], turn, a.wait_limit)) {
                give_up();
                break;
            }
            tmem_fence_after();
            const uint32_t d = tmem + buf * 256 + (static_cast<uint32_t>(32 * quadrant) << 16);
            const int row0 = at.i * GEMM_BM + 32 * quadrant;
            for (int c = 32 * half; c < out_n; c += 64) E::piece(a, g, at.batch, row0, at.j * out_n + c, d + c, st, lane);
            tmem_fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(&taken[buf]);
            buf ^= 1;
            if (buf == 0) turn ^= 1;
        }
        __syncwarp();
    }
    tmem_fence_before();
    __syncthreads();
    if (warp == 2) {
        tmem_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" :: "r"(tmem) : "memory");
    }
}

// ---- host --------------------------------------------------------------------------------------------
// Boxes of 64 x `rows` values (k-major: 64 k of so many rows; m/n-major: 64 columns of so many k) of `batch` matrices of `outer` rows of `inner` 16-bit values.
cudaError_t encode_boxes(CUtensorMap *map, const void *data, bool bf16, int64_t inner, int64_t outer, int64_t batch, int64_t ld, int64_t batch_ld, int rows);

// Whether rows `ld` elements apart from `data` on can be fetched by the copy engine: 16-byte boundaries.
inline bool boxes_fit(const void *data, int64_t ld) { return ((reinterpret_cast<uintptr_t>(data) | static_cast<uintptr_t>(ld * 2)) & 15u) == 0; }

template <typename E>
void begin_gemm(GemmArgs<E> &a, bool bf16, int tile_n, bool dual, bool symmetric, int segments) {
    a.ngroups = a.tiles = 0;
    a.tile_n = tile_n, a.dual = dual, a.symmetric = symmetric, a.segments = segments;
    const int stage = GEMM_A_BYTES + tile_n * GEMM_BK * 2;
    a.stages = (GEMM_SMEM - 1024 - GEMM_EPI_WARPS * GEMM_STAGING) / stage;
    if (a.stages > GEMM_MAX_STAGES) a.stages = GEMM_MAX_STAGES;
    const uint32_t type = bf16 ? 1 : 0;
    a.idesc = 1u << 4 | type << 7 | type << 10 | static_cast<uint32_t>(tile_n >> 3) << 17 | static_cast<uint32_t>(GEMM_BM >> 4) << 24;
}
inline int tiles_of(int m, int n, int tile_n, bool symmetric) {
    const int mt = (m + GEMM_BM - 1) / GEMM_BM, nt = (n + tile_n - 1) / tile_n;
    if (!symmetric) return mt * nt;
    int all = 0;
    for (int i = 0; i < mt; ++i) all += std::min((i * GEMM_BM + GEMM_BM - 1) / tile_n + 1, nt);
    return all;
}
// The next group, of `count` matrices: its sizes and tiles; the rest is the caller's.
template <typename E>
GemmGroup &add_group(GemmArgs<E> &a, int m, int n, int k, int count) {
    GemmGroup &g = a.groups[a.ngroups++];
    g = GemmGroup{};
    const int out_n = a.dual ? a.tile_n / 2 : a.tile_n;
    g.tile0 = a.tiles;
    g.m = m, g.n = n, g.k = k;
    g.mt = (m + GEMM_BM - 1) / GEMM_BM, g.nt = (n + out_n - 1) / out_n;
    g.per = tiles_of(m, n, out_n, a.symmetric);
    a.tiles += g.per * count;
    return g;
}

template <typename E>
cudaError_t launch_gemm(GemmArgs<E> &a, int *err, int wait_limit, cudaStream_t stream, int *launches) {
    if (a.tiles == 0) return cudaSuccess;
    a.err = err, a.wait_limit = wait_limit;
    const size_t smem = 1024 + static_cast<size_t>(a.stages) * (GEMM_A_BYTES + a.tile_n * GEMM_BK * 2) + GEMM_EPI_WARPS * GEMM_STAGING;
    cudaError_t e = cudaFuncSetAttribute(gemm_kernel<E>, cudaFuncAttributeMaxDynamicSharedMemorySize, GEMM_SMEM);
    if (e != cudaSuccess) return e;
    e = launch_op(gemm_kernel<E>, dim3(static_cast<unsigned>(std::min(a.tiles, NUM_SMS))), dim3(GEMM_THREADS), smem, true, stream, a);
    if (e == cudaSuccess) ++*launches;
    return e;
}

}  // namespace desloc
