// The gated feed-forward block of every worker, with its own weights, and its backward pass.
#include "desloc_blocks.cuh"
#include "desloc_gemm.cuh"

#include <type_traits>

namespace desloc {

namespace {

// (Off by 2 + 1.2 |x| units of fp32's last place for the exponential, two for the quotient: 2^-20 near 0, 2^-16 at |x| = 80; the results are rounded to bf16, 2^-8.)
__device__ __forceinline__ float sigmoid(float x) { return __fdividef(1.f, 1.f + __expf(-x)); }

// ---- forward -----------------------------------------------------------------------------------------
// z = silu(g) u of the two halves of the accumulator; g and u, too, where they are kept.  Bound: tensor cores.  4 x 2048 tokens, 2048 x 8192: 440 us for 550 GFLOP.
struct UpEpilogue {
    static constexpr int STAGING = 3 * 2048;
    static constexpr bool READS_BOXES = false, WRITES_BOXES = true;
    struct Ahead {};
    __device__ static bool wants(const GemmGroup &g, int row0, int col0) { return row0 < g.m && col0 < g.n; }
    using Args = GemmArgs<UpEpilogue>;
    __device__ static void fetch(const Args &, const GemmGroup &, int, int, int, int, Ahead &) {}
    __device__ static void settle(const Args &, const GemmGroup &, int, int, int, char *, int, const Ahead &) {}
    __device__ static void drain(const Args &a, const GemmGroup &g, int, int row0, int col0, uint32_t d, char *st, const char *, int lane) {
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {
            float gv[16], uv[16];
            tmem_load16(d + 16 * half, gv);
            tmem_load16(d + a.tile_n / 2 + 16 * half, uv);
            tmem_wait();
            uint32_t w[8];
            if (g.out[1]) {
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = pack_bf16(gv[2 * e], gv[2 * e + 1]);
                put16(st + 2048, lane, half, w);
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = pack_bf16(uv[2 * e], uv[2 * e + 1]);
                put16(st + 4096, lane, half, w);
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) gv[e] = gv[e] * sigmoid(gv[e]) * uv[e];
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = pack_bf16(gv[2 * e], gv[2 * e + 1]);
            put16(st, lane, half, w);
        }
    }
    __device__ static void send_boxes(const Args &a, const GemmGroup &g, int batch, int row0, int col0, const char *st, const char *) {
        for (int k = 0; k < (g.out[1] ? 3 : 1); ++k) tma_store(&a.maps[g.out_map + k], col0, row0, g.io_batch + batch, st + 2048 * k);
    }
    __device__ static void send(const Args &, const GemmGroup &g, int, int row0, int col0, const char *st, int lane) {
        const Piece p = piece_at(g, row0, col0, g.wide & 1), q = piece_at(g, row0, col0, (g.wide & 2) != 0);
        send16(st, lane, static_cast<__nv_bfloat16 *>(g.out[0]) + row0 * g.out_ld + col0, g.out_ld, p);
        if (g.out[1]) {
            const long long kept = row0 * g.in_ld + col0;
            send16(st + 2048, lane, static_cast<__nv_bfloat16 *>(g.out[1]) + kept, g.in_ld, q);
            send16(st + 4096, lane, static_cast<__nv_bfloat16 *>(g.out[2]) + kept, g.in_ld, q);
        }
    }
};

// A product as it is, in bf16 or fp32, or added to what is there.  Bound: tensor cores.  The same sizes: down 216 us for 275 GFLOP, dh 447 for 550, the weights' gradients added to bf16 ones
// 766 for 825.
template <bool BF16, bool ADD>
struct StoreEpilogue {
    static constexpr int STAGING = BF16 ? 2048 : 4096;
    static constexpr bool READS_BOXES = false, WRITES_BOXES = false;
    __device__ static bool wants(const GemmGroup &g, int row0, int col0) { return row0 < g.m && col0 < g.n; }
    struct Was {
        uint4 v[BF16 ? 4 : 8];
    };
    struct Nothing {};
    using Ahead = std::conditional_t<ADD, Was, Nothing>;
    using Args = GemmArgs<StoreEpilogue>;
    __device__ static void fetch(const Args &, const GemmGroup &g, int, int row0, int col0, int lane, Ahead &x) {
        if constexpr (ADD) {
            const Piece p = piece_at(g, row0, col0, g.wide & 1);
            if constexpr (BF16) fetch16(static_cast<const __nv_bfloat16 *>(g.out[0]) + row0 * g.out_ld + col0, g.out_ld, p, lane, x.v);
            else fetch32(static_cast<const float *>(g.out[0]) + row0 * g.out_ld + col0, g.out_ld, p, lane, x.v);
        }
    }
    __device__ static void settle(const Args &, const GemmGroup &g, int, int row0, int col0, char *st, int lane, const Ahead &x) {
        if constexpr (ADD) {
            if constexpr (BF16)
                settle16(st, lane, static_cast<const __nv_bfloat16 *>(g.out[0]) + row0 * g.out_ld + col0, g.out_ld, piece_at(g, row0, col0, g.wide & 1), x.v);
            else settle32(st, lane, x.v);
        }
    }
    __device__ static void drain(const Args &, const GemmGroup &g, int, int row0, int col0, uint32_t d, char *st, const char *, int lane) {
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {
            float v[16];
            tmem_load16(d + 16 * half, v);
            tmem_wait();
            if constexpr (BF16) {
                uint32_t w[8];
                if constexpr (ADD) {
                    row16(st, lane, half, w);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float2 was = unpack_bf16(w[e]);
                        v[2 * e] += was.x, v[2 * e + 1] += was.y;
                    }
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = pack_bf16(v[2 * e], v[2 * e + 1]);
                put16(st, lane, half, w);
            } else {
                if constexpr (ADD) {
                    float was[16];
                    row32(st, lane, half, was);
#pragma unroll
                    for (int e = 0; e < 16; ++e) v[e] += was[e];
                }
                put32(st, lane, half, v);
            }
        }
    }
    __device__ static void send(const Args &, const GemmGroup &g, int, int row0, int col0, const char *st, int lane) {
        const Piece p = piece_at(g, row0, col0, g.wide & 1);
        const long long to = row0 * g.out_ld + col0;
        if constexpr (BF16) send16(st, lane, static_cast<__nv_bfloat16 *>(g.out[0]) + to, g.out_ld, p);
        else send32(st, lane, static_cast<float *>(g.out[0]) + to, g.out_ld, p);
    }
};

// ---- backward ----------------------------------------------------------------------------------------
// From dz = dy down: z = silu(g) u again, du = dz silu(g), dg = dz u (s + silu(g) (1 - s)) with s the sigmoid of g.  Bound: at short k what comes and goes by element, 10 bytes each; 4 x 8192
// tokens, 576 x 1536: 150 us, 3.4 TB/s of those; 4 x 2048, 2048 x 8192: 300 .. 340 us for 275 GFLOP.
struct DzEpilogue {
    static constexpr int STAGING = 3 * 2048;
    static constexpr bool READS_BOXES = false, WRITES_BOXES = true;
    __device__ static bool wants(const GemmGroup &g, int row0, int col0) { return row0 < g.m && col0 < g.n; }
    struct Ahead {
        uint4 g[4], u[4];
    };
    using Args = GemmArgs<DzEpilogue>;
    __device__ static void fetch(const Args &, const GemmGroup &g, int, int row0, int col0, int lane, Ahead &x) {
        const Piece p = piece_at(g, row0, col0, (g.wide & 2) != 0);
        const long long from = row0 * g.in_ld + col0;
        fetch16(static_cast<const __nv_bfloat16 *>(g.in[0]) + from, g.in_ld, p, lane, x.g);
        fetch16(static_cast<const __nv_bfloat16 *>(g.in[1]) + from, g.in_ld, p, lane, x.u);
    }
    __device__ static void settle(const Args &, const GemmGroup &g, int, int row0, int col0, char *st, int lane, const Ahead &x) {
        const Piece p = piece_at(g, row0, col0, (g.wide & 2) != 0);
        const long long from = row0 * g.in_ld + col0;
        settle16(st, lane, static_cast<const __nv_bfloat16 *>(g.in[0]) + from, g.in_ld, p, x.g);
        settle16(st + 2048, lane, static_cast<const __nv_bfloat16 *>(g.in[1]) + from, g.in_ld, p, x.u);
    }
    __device__ static void drain(const Args &, const GemmGroup &g, int, int row0, int col0, uint32_t d, char *st, const char *, int lane) {
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {
            uint32_t gw[8], uw[8], zw[8];
            float v[16];
            tmem_load16(d + 16 * half, v);
            row16(st, lane, half, gw);
            row16(st + 2048, lane, half, uw);
            tmem_wait();
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float2 gg = unpack_bf16(gw[e]), uu = unpack_bf16(uw[e]);
                const float sx = sigmoid(gg.x), sy = sigmoid(gg.y), ax = gg.x * sx, ay = gg.y * sy;
                zw[e] = pack_bf16(ax * uu.x, ay * uu.y);
                gw[e] = pack_bf16(v[2 * e] * uu.x * (sx + ax * (1.f - sx)), v[2 * e + 1] * uu.y * (sy + ay * (1.f - sy)));
                uw[e] = pack_bf16(v[2 * e] * ax, v[2 * e + 1] * ay);
            }
            put16(st, lane, half, gw);
            put16(st + 2048, lane, half, uw);
            put16(st + 4096, lane, half, zw);
        }
    }
    __device__ static void send_boxes(const Args &a, const GemmGroup &g, int batch, int row0, int col0, const char *st, const char *) {
        for (int k = 0; k < 3; ++k) tma_store(&a.maps[g.out_map + k], col0, row0, g.io_batch + batch, st + (k == 0 ? 4096 : 2048 * (k - 1)));
    }
    __device__ static void send(const Args &, const GemmGroup &g, int, int row0, int col0, const char *st, int lane) {
        const Piece p = piece_at(g, row0, col0, g.wide & 1);
        const long long to = row0 * g.out_ld + col0;
        send16(st + 4096, lane, static_cast<__nv_bfloat16 *>(g.out[0]) + to, g.out_ld, p);
        send16(st, lane, static_cast<__nv_bfloat16 *>(g.out[1]) + to, g.out_ld, p);
        send16(st + 2048, lane, static_cast<__nv_bfloat16 *>(g.out[2]) + to, g.out_ld, p);
    }
};

// ---- single tokens -----------------------------------------------------------------------------------
// Up to FFN_FEW tokens of a worker: a warp for each row of the weights, which it reads from one end to the other.  Bound: HBM, the weights once.  (Tiles of the tensor cores
// bring 128 bytes of many rows at a time, for which memory is slower.  Four workers, one token, width 2048, hidden 8192, 403 MB: 67 us, 6.0 TB/s, 0.92 of copy; by tiles
// 92 us.)  Sums in fp32, lanes' sums in a fixed order.
// Tiles take the same for 1 to 64 tokens, rows longer with each (every warp reads the tokens' values again).  Rows at 1 / 2 / 3 / 4 / 5 / 8 tokens against tiles: four workers, 2048 x
// 8192, 68 / 78 / 83 / 99 / 125 / 188 us against 92; eight, 960 x 2560, 25 / 30 / 34 / 40 / 50 / 75 against 38; four, 576 x 1536, 9 / 10 / 11 / 13 / 15 / 22 against 23.  So at four
// tokens rows lose 5 to 8 % in large blocks and win 44 % in small ones; at five they lose a third in large ones.
constexpr int FFN_FEW = 4, FEW_THREADS = 256, FEW_AHEAD = 4;

// Sums of a row of w (and, where W = 2, of a second one) times T rows of x, of which the next one is x_ld further on.
template <int W, int T>
__device__ __forceinline__ void dots(const __nv_bfloat16 *const (&w)[W], const __nv_bfloat16 *x, long long x_ld, int k, float (&sum)[W][T]) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int i = 0; i < W; ++i)
#pragma unroll
        for (int t = 0; t < T; ++t) sum[i][t] = 0.f;
    uintptr_t low = reinterpret_cast<uintptr_t>(x) | static_cast<uintptr_t>(T > 1 ? x_ld * 2 : 0) | static_cast<uintptr_t>(k * 2);
    for (const __nv_bfloat16 *p : w) low |= reinterpret_cast<uintptr_t>(p);
    if (low % 16 == 0) {
        for (int c = 8 * lane; c < k; c += 256 * FEW_AHEAD) {
            uint4 v[FEW_AHEAD][W];
#pragma unroll
            for (int a = 0; a < FEW_AHEAD; ++a)
#pragma unroll
                for (int i = 0; i < W; ++i) v[a][i] = c + 256 * a < k ? __ldcs(reinterpret_cast<const uint4 *>(w[i] + c + 256 * a)) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int a = 0; a < FEW_AHEAD; ++a) {
                if (c + 256 * a >= k) break;
                float f[W][8];
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    const uint32_t h[4] = {v[a][i].x, v[a][i].y, v[a][i].z, v[a][i].w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float2 two = unpack_bf16(h[e]);
                        f[i][2 * e] = two.x, f[i][2 * e + 1] = two.y;
                    }
                }
#pragma unroll
                for (int t = 0; t < T; ++t) {
                    float y[8];
                    load_values(x + t * x_ld + c + 256 * a, y);
#pragma unroll
                    for (int i = 0; i < W; ++i)
#pragma unroll
                        for (int e = 0; e < 8; ++e) sum[i][t] = fmaf(f[i][e], y[e], sum[i][t]);
                }
            }
        }
    } else {
#pragma unroll 4
        for (int c = lane; c < k; c += 32)
#pragma unroll
            for (int t = 0; t < T; ++t) {
                const float y = __bfloat162float(x[t * x_ld + c]);
#pragma unroll
                for (int i = 0; i < W; ++i) sum[i][t] = fmaf(__bfloat162float(w[i][c]), y, sum[i][t]);
            }
    }
#pragma unroll
    for (int i = 0; i < W; ++i)
#pragma unroll
        for (int t = 0; t < T; ++t)
#pragma unroll
            for (int d = 16; d; d /= 2) sum[i][t] += __shfl_xor_sync(0xffffffffu, sum[i][t], d);
}

template <int T>
__global__ void __launch_bounds__(FEW_THREADS, T <= 2 ? 4 : 3) ffn_few_up_kernel(const __grid_constant__ FfnArgs a, __nv_bfloat16 *z) {
    begin_and_let_next_begin();
    const int m = blockIdx.y, j = blockIdx.x * (FEW_THREADS / 32) + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    wait_for_earlier_kernels();
    if (j >= a.hidden) return;
    const long long at = static_cast<long long>(j) * a.width;
    const __nv_bfloat16 *const w[2] = {static_cast<const __nv_bfloat16 *>(a.gate[m]) + at, static_cast<const __nv_bfloat16 *>(a.up[m]) + at};
    float sum[2][T];
    dots<2, T>(w, static_cast<const __nv_bfloat16 *>(a.h) + m * a.hs0, a.hs1, a.width, sum);
#pragma unroll
    for (int t = 0; t < T; ++t)
        if (lane == t) {
            const long long to = (static_cast<long long>(m) * T + t) * a.hidden + j;
            z[to] = __float2bfloat16_rn(sum[0][t] * sigmoid(sum[0][t]) * sum[1][t]);
            if (a.kept_gate) {
                static_cast<__nv_bfloat16 *>(a.kept_gate)[to] = __float2bfloat16_rn(sum[0][t]);
                static_cast<__nv_bfloat16 *>(a.kept_up)[to] = __float2bfloat16_rn(sum[1][t]);
            }
        }
}

template <int T>
__global__ void __launch_bounds__(FEW_THREADS, T <= 2 ? 4 : 3) ffn_few_down_kernel(const __grid_constant__ FfnArgs a, const __nv_bfloat16 *z) {
    begin_and_let_next_begin();
    const int m = blockIdx.y, j = blockIdx.x * (FEW_THREADS / 32) + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    wait_for_earlier_kernels();
    if (j >= a.width) return;
    const __nv_bfloat16 *const w[1] = {static_cast<const __nv_bfloat16 *>(a.down[m]) + static_cast<long long>(j) * a.hidden};
    float sum[1][T];
    dots<1, T>(w, z + static_cast<long long>(m) * T * a.hidden, a.hidden, a.hidden, sum);
#pragma unroll
    for (int t = 0; t < T; ++t)
        if (lane == t) static_cast<__nv_bfloat16 *>(a.y)[m * a.ys0 + t * a.ys1 + j] = __float2bfloat16_rn(sum[0][t]);
}

template <int T>
cudaError_t launch_few(const FfnArgs &a, __nv_bfloat16 *z, cudaStream_t stream, int *launches) {
    const auto blocks = [&](int n) { return dim3((n + FEW_THREADS / 32 - 1) / (FEW_THREADS / 32), a.M); };
    cudaError_t e = launch_op(ffn_few_up_kernel<T>, blocks(a.hidden), dim3(FEW_THREADS), 0, true, stream, a, z);
    if (e == cudaSuccess) ++*launches, e = launch_op(ffn_few_down_kernel<T>, blocks(a.width), dim3(FEW_THREADS), 0, true, stream, a, z);
    if (e == cudaSuccess) ++*launches;
    return e;
}

// ---- rows that the copy engine does not take ---------------------------------------------------------
// Copies matrices into rows on 16-byte boundaries.  Bound: HBM, two bytes each way; 4 x 3 matrices of 1501 x 4003 in 68 us, 4.2 TB/s.  A warp takes a row, a lane 16 bytes of the copy, which lie in two aligned
// pieces of 16 bytes.
constexpr int PACK_MOST = 64;
struct PackArgs {
    const unsigned short *from[PACK_MOST];
    unsigned short *to;
    long long from_ld, to_ld, to_batch;
    int rows, cols;
};
__global__ void __launch_bounds__(256) pack_kernel(const __grid_constant__ PackArgs a) {
    begin_and_let_next_begin();
    wait_for_earlier_kernels();
    const unsigned short *from = a.from[blockIdx.y];
    unsigned short *to = a.to + blockIdx.y * a.to_batch;
    const int lane = threadIdx.x & 31;
    for (long long r = blockIdx.x * 8ll + (threadIdx.x >> 5); r < a.rows; r += gridDim.x * 8ll) {
        const unsigned short *const row = from + r * a.from_ld;
        const int off = static_cast<int>(reinterpret_cast<uintptr_t>(row) & 15);   // bytes, even
        const uint4 *const pieces = reinterpret_cast<const uint4 *>(reinterpret_cast<uintptr_t>(row) - off);
        const int chunks = a.cols / 8, last = (off + 2 * a.cols) / 16;   // whole ones of the copy; aligned pieces [first, last) lie in the row
        const int first = off ? 1 : 0;
        constexpr int AHEAD = 4;
        for (int c0 = lane; c0 < chunks; c0 += 32 * AHEAD) {
            uint4 v[AHEAD], n[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const int c = c0 + 32 * k;
                const bool whole = c >= first && c + first < last;   // all of its pieces lie in the row
                v[k] = whole ? pieces[c] : make_uint4(0, 0, 0, 0);
                n[k] = whole && off ? pieces[c + 1] : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const int c = c0 + 32 * k;
                if (c >= chunks) break;
                unsigned short *const out = to + r * a.to_ld + 8 * c;
                if (c < first || c + first >= last) {
                    for (int e = 0; e < 8; ++e) out[e] = row[8 * c + e];
                    continue;
                }
                uint32_t w[8] = {v[k].x, v[k].y, v[k].z, v[k].w, n[k].x, n[k].y, n[k].z, n[k].w};
                if (off & 8) {
#pragma unroll
                    for (int e = 0; e < 6; ++e) w[e] = w[e + 2];
                }
                if (off & 4) {
#pragma unroll
                    for (int e = 0; e < 5; ++e) w[e] = w[e + 1];
                }
                if (off & 2) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[e] = __funnelshift_r(w[e], w[e + 1], 16);
                }
                *reinterpret_cast<uint4 *>(out) = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
        for (int e = 8 * chunks + lane; e < a.cols; e += 32) to[r * a.to_ld + e] = row[e];
    }
}

int64_t padded(int64_t n) { return (n + 7) & ~int64_t{7}; }

// An operand of every worker's: where it lies, or where it is copied to.
struct Operand {
    bool batched;               // one map for all workers, at `data`
    const void *data;
    const void *const *each;    // or an address per worker
    int64_t rows, cols, ld, batch_ld;
    bool packed;
    int64_t bytes;              // of the copy

    static Operand rows_of(const void *data, int M, int64_t rows, int64_t cols, long long s0, long long s1) {
        Operand o{true, data, nullptr, rows, cols, rows == 1 ? padded(cols) : s1, M == 1 ? padded(cols) * rows : s0, false, 0};
        o.packed = !boxes_fit(data, o.ld) || !boxes_fit(data, o.batch_ld) || o.ld < cols || o.batch_ld < 1 || o.ld >= (1ll << 38) || o.batch_ld >= (1ll << 38);
        if (o.packed) o.bytes = M * rows * padded(cols) * 2;
        return o;
    }
    static Operand weights(const void *const *each, int M, int64_t rows, int64_t cols) {
        Operand o{false, nullptr, each, rows, cols, cols, 0, false, 0};
        for (int m = 0; m < M; ++m) o.packed = o.packed || !boxes_fit(each[m], cols);
        if (o.packed) o.bytes = M * rows * padded(cols) * 2;
        return o;
    }
    // Fetches the operand of the workers [m0, m0 + n) in boxes of `box_rows`: from map `first` on, one map for all or one each.
    template <typename E>
    cudaError_t maps(GemmArgs<E> &a, int first, int every, int M, int m0, int n, int box_rows) const {
        if (batched) return encode_boxes(&a.maps[first], data, true, cols, rows, M, ld, batch_ld, box_rows);
        for (int i = 0; i < n; ++i) {
            const cudaError_t e = encode_boxes(&a.maps[first + i * every], each[m0 + i], true, cols, rows, 1, ld, padded(cols) * rows, box_rows);
            if (e != cudaSuccess) return e;
        }
        return cudaSuccess;
    }
};

struct Bump {
    char *work;
    int64_t used = 0;
    void *take(int64_t bytes) {
        char *p = work ? work + used : nullptr;
        used += (bytes + 255) & ~int64_t{255};
        return p;
    }
};

// Copies an operand where it has to be, and says where it is from then on.
cudaError_t pack(Operand &o, int M, long long s0, long long s1, Bump &bump, cudaStream_t stream, int *launches) {
    if (!o.packed) return cudaSuccess;
    PackArgs a{};
    a.to = static_cast<unsigned short *>(bump.take(o.bytes));
    a.rows = static_cast<int>(o.rows), a.cols = static_cast<int>(o.cols);
    a.from_ld = o.batched ? s1 : o.ld;
    a.to_ld = padded(o.cols), a.to_batch = o.rows * a.to_ld;
    const unsigned short *const base = static_cast<const unsigned short *>(o.data);
    unsigned short *const start = a.to;
    for (int m0 = 0; m0 < M; m0 += PACK_MOST) {
        const int n = std::min(PACK_MOST, M - m0);
        for (int i = 0; i < n; ++i) a.from[i] = o.batched ? base + (m0 + i) * s0 : static_cast<const unsigned short *>(o.each[m0 + i]);
        a.to = start + m0 * a.to_batch;
        const unsigned blocks = static_cast<unsigned>(std::min<int64_t>((o.rows + 7) / 8, std::max(1, 8 * NUM_SMS / n)));
        const cudaError_t e = launch_op(pack_kernel, dim3(blocks, n), dim3(256), 0, true, stream, a);
        if (e != cudaSuccess) return e;
        ++*launches;
    }
    o.batched = true, o.data = start, o.ld = a.to_ld, o.batch_ld = a.to_batch;
    return cudaSuccess;
}

// Results leave as boxes where emptying a tile takes longer than its products, in which the copy engine has more to do: products of up to BOXES_K (8192 x 576 x 1536 by four
// workers 173 us instead of 194; 2048 x 2048 x 8192 304 us instead of 293).  The whole way back with / without them, four workers, two runs each, us: 8192 tokens of width 576 419, 419 /
// 440, 445; 4096 of 768 299, 299 / 310, 312; of 960 464, 474 / 479, 480; of 1024 720, 740 / 748, 862; of 1280 886, 787 / 796, 867; 2048 of 1536 519, 524 / 526, 526; of 2048 1407,
// 1409 / 1361, 1423: beyond 1024 no difference that lasts.  The way forward takes 0 to 2 % longer with boxes at all of these.
constexpr int BOXES_K = 1024;
constexpr int WORKERS = 16;   // of a launch: three groups and two maps each at most

struct Run {
    cudaStream_t stream;
    int *err, wait_limit, *launches;
};

bool wide16(const void *p, long long ld) { return boxes_fit(p, ld); }
bool wide32(const void *p, long long ld) { return ((reinterpret_cast<uintptr_t>(p) | static_cast<uintptr_t>(ld * 4)) & 15u) == 0; }

cudaError_t product_store(const Operand &x, const Operand &w, int M, int tokens, int n, int k, void *out, long long s0, long long s1, const Run &r) {
    using E = StoreEpilogue<true, false>;
    static thread_local GemmArgs<E> a;
    for (int m0 = 0; m0 < M; m0 += WORKERS) {
        const int some = std::min(WORKERS, M - m0);
        const GemmCut cut = pick_cut(false, tokens, k, [&](const GemmCut &c) { return TileCount{static_cast<int64_t>(some) * tiles_of(tokens, n, c, false, false), 0}; });
        begin_gemm(a, true, cut, false, false, 1);
        cudaError_t e = x.maps(a, 0, 0, M, m0, some, box_rows(tokens));
        if (e == cudaSuccess) e = w.maps(a, 1, 1, M, m0, some, cut.box_n(false));
        if (e != cudaSuccess) return e;
        for (int i = 0; i < some; ++i) {
            GemmGroup &g = add_group(a, tokens, n, k, 1);
            g.a_map = 0, g.a_batch = m0 + i;
            g.b_map = static_cast<short>(w.batched ? 1 : 1 + i), g.b_batch = w.batched ? m0 + i : 0;
            g.out[0] = static_cast<__nv_bfloat16 *>(out) + (m0 + i) * s0;
            g.out_ld = s1;
            g.wide = wide16(g.out[0], s1);
        }
        e = launch_gemm(a, r.err, r.wait_limit, r.stream, r.launches);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

struct Operands {
    Operand h, dy, gate, up, down;
    Operands(const FfnArgs &a, bool backward)
        : h(Operand::rows_of(a.h, a.M, a.tokens, a.width, a.hs0, a.hs1)),
          dy(backward ? Operand::rows_of(a.dy, a.M, a.tokens, a.width, a.dys0, a.dys1) : Operand{}),
          gate(Operand::weights(a.gate, a.M, a.hidden, a.width)), up(Operand::weights(a.up, a.M, a.hidden, a.width)),
          down(Operand::weights(a.down, a.M, a.width, a.hidden)) {}
    cudaError_t pack_all(const FfnArgs &a, bool backward, Bump &bump, const Run &r) {
        cudaError_t e = pack(h, a.M, a.hs0, a.hs1, bump, r.stream, r.launches);
        if (e == cudaSuccess && backward) e = pack(dy, a.M, a.dys0, a.dys1, bump, r.stream, r.launches);
        for (Operand *o : {&gate, &up, &down})
            if (e == cudaSuccess) e = pack(*o, a.M, 0, 0, bump, r.stream, r.launches);
        return e;
    }
};

// A k- or m/n-major operand of `rows` token rows in working memory.
Operand inner_operand(const void *data, const FfnArgs &a, int64_t cols) {
    return Operand::rows_of(data, a.M, a.tokens, cols, a.tokens * padded(cols), padded(cols));
}

template <bool BF16, bool ADD>
cudaError_t weight_grads(const FfnArgs &a, const Operands &o, const Operand &z, const Operand &dg, const Operand &du, const Run &r) {
    using E = StoreEpilogue<BF16, ADD>;
    static thread_local GemmArgs<E> g;
    for (int m0 = 0; m0 < a.M; m0 += WORKERS) {
        const int some = std::min(WORKERS, a.M - m0);
        const GemmCut cut = pick_cut(false, GEMM_BM, a.tokens, [&](const GemmCut &c) {
            return TileCount{static_cast<int64_t>(some) * (2 * tiles_of(a.hidden, a.width, c, false, false) + tiles_of(a.width, a.hidden, c, false, false)), 0};
        });
        begin_gemm(g, true, cut, false, false, 1);
        int map = 0;
        for (const Operand *x : {&dg, &du, &o.dy, &o.h, &z}) {
            const cudaError_t e = x->maps(g, map++, 0, a.M, m0, some, 64);
            if (e != cudaSuccess) return e;
        }
        for (int which = 0; which < 3; ++which)
            for (int i = 0; i < some; ++i) {
                GemmGroup &group = which < 2 ? add_group(g, a.hidden, a.width, a.tokens, 1) : add_group(g, a.width, a.hidden, a.tokens, 1);
                group.a_map = static_cast<short>(which), group.b_map = which < 2 ? 3 : 4;
                group.a_mn = group.b_mn = 1;
                group.a_batch = group.b_batch = m0 + i;
                group.out[0] = which == 0 ? a.dgate[m0 + i] : which == 1 ? a.dup[m0 + i] : a.ddown[m0 + i];
                group.out_ld = which < 2 ? a.width : a.hidden;
                group.wide = BF16 ? wide16(group.out[0], group.out_ld) : wide32(group.out[0], group.out_ld);
            }
        const cudaError_t e = launch_gemm(g, r.err, r.wait_limit, r.stream, r.launches);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace

int64_t ffn_work(const FfnArgs &a, bool backward) {
    Bump bump{nullptr};
    const Operands o(a, backward);
    if (backward || a.tokens > FFN_FEW)
        for (const Operand *x : {&o.h, &o.dy, &o.gate, &o.up, &o.down}) bump.take(x->bytes);
    for (int i = 0; i < (backward ? 3 : 1); ++i) bump.take(static_cast<int64_t>(a.M) * a.tokens * padded(a.hidden) * 2);
    return bump.used;
}

cudaError_t launch_ffn(const FfnArgs &a, char *work, int *err, int wait_limit, cudaStream_t stream, int *launches) {
    const Run r{stream, err, wait_limit, launches};
    Bump bump{work};
    if (a.tokens <= FFN_FEW) {
        __nv_bfloat16 *const few = static_cast<__nv_bfloat16 *>(bump.take(static_cast<int64_t>(a.M) * a.tokens * a.hidden * 2));
        return (a.tokens == 1 ? launch_few<1> : a.tokens == 2 ? launch_few<2> : a.tokens == 3 ? launch_few<3> : launch_few<4>)(a, few, stream, launches);
    }
    Operands o(a, false);
    const long long ld = padded(a.hidden), per = a.tokens * ld;
    __nv_bfloat16 *const z = static_cast<__nv_bfloat16 *>(bump.take(a.M * per * 2));
    cudaError_t e = o.pack_all(a, false, bump, r);
    if (e != cudaSuccess) return e;
    static thread_local GemmArgs<UpEpilogue> g;
    for (int m0 = 0; m0 < a.M; m0 += WORKERS) {
        const int some = std::min(WORKERS, a.M - m0);
        const GemmCut cut = pick_cut(true, a.tokens, a.width, [&](const GemmCut &c) { return TileCount{static_cast<int64_t>(some) * tiles_of(a.tokens, a.hidden, c, true, false), 0}; });
        const int box = cut.box_n(true);
        begin_gemm(g, true, cut, true, false, 1);
        e = o.h.maps(g, 0, 0, a.M, m0, some, box_rows(a.tokens));
        // (gate and up of a worker next to one another: the second half of a tile's columns is the next map's)
        if (e == cudaSuccess) e = o.gate.maps(g, 1, 2, a.M, m0, some, box);
        if (e == cudaSuccess) e = o.up.maps(g, 2, 2, a.M, m0, some, box);
        if (e != cudaSuccess) return e;
        // where the one is a single map and the other one each, both take one each
        const bool batched = o.gate.batched && o.up.batched;
        if (!batched) {
            for (int half = 0; half < 2; ++half) {
                const Operand &w = half ? o.up : o.gate;
                if (!w.batched) continue;
                for (int i = 0; i < some && e == cudaSuccess; ++i)
                    e = encode_boxes(&g.maps[1 + half + 2 * i], static_cast<const __nv_bfloat16 *>(w.data) + (m0 + i) * w.batch_ld, true, w.cols, w.rows, 1, w.ld,
                                     w.batch_ld, box);
            }
            if (e != cudaSuccess) return e;
        }
        // z, and g and u where they are kept and lie so, leave as boxes
        const int boxes = 1 + 2 * WORKERS;
        bool whole = a.width <= BOXES_K;
        for (int k = 0; k < (a.kept_gate ? 3 : 1) && whole; ++k) {
            const void *const to = k == 0 ? z : k == 1 ? a.kept_gate : a.kept_up;
            const long long to_ld = k == 0 ? ld : a.hidden;
            whole = boxes_fit(to, to_ld);
            if (whole) e = encode_boxes(&g.maps[boxes + k], to, true, a.hidden, a.tokens, a.M, to_ld, a.tokens * to_ld, 32, 32);
            if (e != cudaSuccess) return e;
        }
        for (int i = 0; i < some; ++i) {
            const int m = m0 + i;
            GemmGroup &group = add_group(g, a.tokens, a.hidden, a.width, 1);
            if (whole) group.out_map = static_cast<short>(boxes), group.io_batch = m;
            group.a_batch = m;
            group.b_map = static_cast<short>(batched ? 1 : 1 + 2 * i), group.b_batch = batched ? m : 0;
            group.out[0] = z + m * per, group.out_ld = ld;
            group.wide = 1;
            if (a.kept_gate) {
                const long long from = static_cast<long long>(m) * a.tokens * a.hidden;
                group.out[1] = static_cast<__nv_bfloat16 *>(a.kept_gate) + from;
                group.out[2] = static_cast<__nv_bfloat16 *>(a.kept_up) + from;
                group.in_ld = a.hidden;
                if (wide16(group.out[1], a.hidden) && wide16(group.out[2], a.hidden)) group.wide |= 2;
            }
        }
        e = launch_gemm(g, err, wait_limit, stream, launches);
        if (e != cudaSuccess) return e;
    }
    return product_store(inner_operand(z, a, a.hidden), o.down, a.M, a.tokens, a.width, a.hidden, a.y, a.ys0, a.ys1, r);
}

cudaError_t launch_ffn_grad(const FfnArgs &a, char *work, int *err, int wait_limit, cudaStream_t stream, int *launches) {
    const Run r{stream, err, wait_limit, launches};
    Bump bump{work};
    Operands o(a, true);
    const long long ld = padded(a.hidden), per = a.tokens * ld;
    __nv_bfloat16 *inner[3];
    for (auto &p : inner) p = static_cast<__nv_bfloat16 *>(bump.take(a.M * per * 2));
    cudaError_t e = o.pack_all(a, true, bump, r);
    if (e != cudaSuccess) return e;
    {
        static thread_local GemmArgs<DzEpilogue> g;
        for (int m0 = 0; m0 < a.M; m0 += WORKERS) {
            const int some = std::min(WORKERS, a.M - m0);
            const GemmCut cut = pick_cut(false, a.tokens, a.width, [&](const GemmCut &c) { return TileCount{static_cast<int64_t>(some) * tiles_of(a.tokens, a.hidden, c, false, false), 0}; });
            begin_gemm(g, true, cut, false, false, 1);
            e = o.dy.maps(g, 0, 0, a.M, m0, some, box_rows(a.tokens));
            if (e == cudaSuccess) e = o.down.maps(g, 1, 1, a.M, m0, some, 64);
            const int boxes = 1 + WORKERS;
            for (int k = 0; k < 3 && e == cudaSuccess && a.width <= BOXES_K; ++k)
                e = encode_boxes(&g.maps[boxes + k], inner[k], true, a.hidden, a.tokens, a.M, ld, per, 32, 32);
            if (e != cudaSuccess) return e;
            for (int i = 0; i < some; ++i) {
                const int m = m0 + i;
                GemmGroup &group = add_group(g, a.tokens, a.hidden, a.width, 1);
                group.a_batch = m;
                group.b_map = static_cast<short>(o.down.batched ? 1 : 1 + i), group.b_batch = o.down.batched ? m : 0;
                group.b_mn = 1;
                const long long from = static_cast<long long>(m) * a.tokens * a.hidden;
                group.in[0] = static_cast<const __nv_bfloat16 *>(a.was_gate) + from;
                group.in[1] = static_cast<const __nv_bfloat16 *>(a.was_up) + from;
                group.in_ld = a.hidden;
                for (int k = 0; k < 3; ++k) group.out[k] = inner[k] + m * per;
                if (a.width <= BOXES_K) group.out_map = static_cast<short>(boxes), group.io_batch = m;
                group.out_ld = ld;
                group.wide = 1 | (wide16(group.in[0], a.hidden) && wide16(group.in[1], a.hidden) ? 2 : 0);
            }
            e = launch_gemm(g, err, wait_limit, stream, launches);
            if (e != cudaSuccess) return e;
        }
    }
    const Operand z = inner_operand(inner[0], a, a.hidden), dg = inner_operand(inner[1], a, a.hidden), du = inner_operand(inner[2], a, a.hidden);
    // (before dh, which may come in the place of h or dy)
    if (a.grad_bf16) e = (a.accumulate ? weight_grads<true, true> : weight_grads<true, false>)(a, o, z, dg, du, r);
    else e = (a.accumulate ? weight_grads<false, true> : weight_grads<false, false>)(a, o, z, dg, du, r);
    if (e != cudaSuccess) return e;
    {
        // dh = dg gate + du up, one accumulator
        using E = StoreEpilogue<true, false>;
        static thread_local GemmArgs<E> g;
        for (int m0 = 0; m0 < a.M; m0 += WORKERS) {
            const int some = std::min(WORKERS, a.M - m0);
            const GemmCut cut = pick_cut(false, a.tokens, 2 * a.hidden, [&](const GemmCut &c) { return TileCount{static_cast<int64_t>(some) * tiles_of(a.tokens, a.width, c, false, false), 0}; });
            begin_gemm(g, true, cut, false, false, 2);
            e = dg.maps(g, 0, 0, a.M, m0, some, box_rows(a.tokens));
            if (e == cudaSuccess) e = du.maps(g, 1, 0, a.M, m0, some, box_rows(a.tokens));
            for (int i = 0; i < some && e == cudaSuccess; ++i)
                for (int seg = 0; seg < 2 && e == cudaSuccess; ++seg) {
                    const Operand &w = seg ? o.up : o.gate;
                    const void *from = w.batched ? static_cast<const __nv_bfloat16 *>(w.data) + (m0 + i) * w.batch_ld : w.each[m0 + i];
                    e = encode_boxes(&g.maps[2 + 2 * i + seg], from, true, w.cols, w.rows, 1, w.ld, padded(w.cols) * w.rows, 64);
                }
            if (e != cudaSuccess) return e;
            for (int i = 0; i < some; ++i) {
                GemmGroup &group = add_group(g, a.tokens, a.width, a.hidden, 1);
                group.a_batch = m0 + i;
                group.b_map = static_cast<short>(2 + 2 * i), group.b_mn = 1;
                group.out[0] = static_cast<__nv_bfloat16 *>(a.dh) + (m0 + i) * a.dhs0;
                group.out_ld = a.dhs1;
                group.wide = wide16(group.out[0], a.dhs1);
            }
            e = launch_gemm(g, err, wait_limit, stream, launches);
            if (e != cudaSuccess) return e;
        }
    }
    return cudaSuccess;
}

}  // namespace desloc
