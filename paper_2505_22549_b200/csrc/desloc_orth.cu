// Orthogonalised updates: Newton-Schulz products of every worker's matrices, from the momentum to the step.
#include "desloc_blocks.cuh"
#include "desloc_gemm.cuh"

#include <algorithm>

namespace desloc {

namespace {

// X := U / (|U| + eps), then `steps` times X := a X + (b G + c G^2) X with G = X X^T (of tall matrices: X := a X + X (b G + c G^2), G = X^T X, the same
// by the shorter side).  Each step is three products: G and G^2 are symmetric, of them the lower triangle is computed and written to both places.
//
// Operands are fp16: with bf16's eight bits the result was off by 1 % of its norm (normal 576 x 1536 matrices) and by 10 % and more where few directions dominate,
// since a step takes small singular values times a = 3.4 and the rounding errors next to them too.  X is carried as two fp16 numbers (hi + lo / 2^11, 22 bits): hi is
// the operand, a X takes both (a is on the diagonal of the polynomial, a lo is added behind the product), so that what is rounded away in one step is there in the
// next.  Off by 0.15 % for normal matrices, 0.03 % for few directions.
// Everything is held times ORTH_UNIT: singular values stay below two, entries far below one.
constexpr float ORTH_UNIT = 256.f, ORTH_LO = 2048.f;
constexpr int ORTH_ROUND = 512, ORTH_SHAPES = 16;   // matrices and shapes of one round of launches
constexpr int ORTH_THREADS = 256, ORTH_WARPS = ORTH_THREADS / 32;

struct Sources {
    const void *update[ORTH_ROUND];   // null: table[index]
    const void *grad[ORTH_ROUND];     // null: none
    int index[ORTH_ROUND];
    int shape[ORTH_ROUND];
    int number[ORTH_ROUND];           // of those of its shape
    struct {
        int rows, cols, ld, block_rows;
        __half *hi, *lo;              // of the shape's first matrix
    } shapes[ORTH_SHAPES];
    float *const *table;
    double *partial;                  // [matrices][most]
    int most;
    float beta, eps, rho;
};

// N values as they lie in memory: they wait in as few registers as they can, since how many are on their way is what the bandwidth comes from.
template <typename T, int N>
struct Raw {
    uint4 q[N * sizeof(T) / 16];
    __device__ __forceinline__ void load(const T *p) {
#pragma unroll
        for (int i = 0; i < static_cast<int>(N * sizeof(T) / 16); ++i) q[i] = reinterpret_cast<const uint4 *>(p)[i];
    }
    __device__ __forceinline__ void values(float (&f)[N]) const {
#pragma unroll
        for (int i = 0; i < static_cast<int>(N * sizeof(T) / 16); ++i) {
            const uint32_t w[4] = {q[i].x, q[i].y, q[i].z, q[i].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (sizeof(T) == 4) {
                    f[4 * i + e] = __uint_as_float(w[e]);
                } else {
                    const float2 two = unpack_bf16(w[e]);
                    f[8 * i + 2 * e] = two.x, f[8 * i + 2 * e + 1] = two.y;
                }
            }
        }
    }
};
template <typename T>
struct Raw<T, 1> {
    T v;
    __device__ __forceinline__ void load(const T *p) { v = *p; }
    __device__ __forceinline__ void values(float (&f)[1]) const { f[0] = static_cast<float>(v); }
};

// The elements that a block of a matrix takes (they follow one another), as fp32: f(first one's number within the block, values) for N of them at a time, AHEAD times as
// many on their way per thread; N = 8 where rows and addresses allow it.
template <typename UT, typename GT, typename F>
__device__ __forceinline__ void visit(const Sources &s, int which, long long first, int count, const F &f) {
    const UT *const u = static_cast<const UT *>(s.update[which] ? s.update[which] : s.table[s.index[which]]) + first;
    const GT *const g = s.grad[which] ? static_cast<const GT *>(s.grad[which]) + first : nullptr;
    const float beta = s.beta, rest = 1.f - s.beta, rho = s.rho;
    const auto go = [&](auto width, auto ahead) {
        constexpr int N = decltype(width)::value, STEP = ORTH_THREADS * N;
        constexpr bool WITH = decltype(ahead)::value;   // with gradients
        constexpr int AHEAD = N == 1 ? 8 : sizeof(UT) == 2 && !WITH ? 4 : 2;
        for (int at = threadIdx.x * N; at < count; at += STEP * AHEAD) {
            Raw<UT, N> x[AHEAD];
            Raw<GT, N> y[WITH ? AHEAD : 1];
#pragma unroll
            for (int e = 0; e < AHEAD; ++e)
                if (at + e * STEP < count) x[e].load(u + at + e * STEP);
            if constexpr (WITH) {
#pragma unroll
                for (int e = 0; e < AHEAD; ++e)
                    if (at + e * STEP < count) y[e].load(g + at + e * STEP);
            }
#pragma unroll
            for (int e = 0; e < AHEAD; ++e) {
                if (at + e * STEP >= count) break;
                float v[N];
                x[e].values(v);
                if constexpr (WITH) {
                    float w[N];
                    y[e].values(w);
#pragma unroll
                    for (int k = 0; k < N; ++k) v[k] = beta * v[k] + rest * clipped(w[k], rho);
                }
                f(at + e * STEP, v);
            }
        }
    };
    const bool wide = s.shapes[s.shape[which]].cols % 8 == 0 && ((reinterpret_cast<uintptr_t>(u) | reinterpret_cast<uintptr_t>(g)) & 15) == 0;
    using Wide = std::integral_constant<int, 8>;
    using One = std::integral_constant<int, 1>;
    if (g) wide ? go(Wide(), std::true_type()) : go(One(), std::true_type());
    else wide ? go(Wide(), std::false_type()) : go(One(), std::false_type());
}

__device__ __forceinline__ double block_sum(double v) {
    __shared__ double sums[ORTH_WARPS];
#pragma unroll
    for (int d = 16; d; d /= 2) v += __shfl_xor_sync(0xffffffffu, v, d);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < ORTH_WARPS; ++w) v += sums[w];
    return v;
}

// Squares, eight at a time in fp32 (values below 1e-22 count as 0, beyond 1e18 as infinite), then in fp64.  Bound: HBM, each element read once; 57 M of fp32 with bf16 gradients
// 55 us, 6.2 TB/s.
template <typename UT, typename GT>
__global__ void __launch_bounds__(ORTH_THREADS, 4) orth_norm_kernel(const __grid_constant__ Sources s) {
    begin_and_let_next_begin();
    wait_for_earlier_kernels();
    const int which = blockIdx.y;
    const auto &sh = s.shapes[s.shape[which]];
    const long long first = static_cast<long long>(blockIdx.x) * sh.block_rows * sh.cols;
    const int count = static_cast<int>(min(static_cast<long long>(sh.block_rows) * sh.cols, static_cast<long long>(sh.rows) * sh.cols - first));
    if (count <= 0) return;
    double sum = 0;
    visit<UT, GT>(s, which, first, count, [&](int, const auto &v) {
        float part = 0;
#pragma unroll
        for (float x : v) part += x * x;
        sum += part;
    });
    sum = block_sum(sum);
    if (threadIdx.x == 0) s.partial[static_cast<long long>(which) * s.most + blockIdx.x] = sum;
}

// X in two halves.  Bound: HBM, each element read again and four bytes written; the same 57 M 87 us, 6.5 TB/s.
template <typename UT, typename GT>
__global__ void __launch_bounds__(ORTH_THREADS, 4) orth_scale_kernel(const __grid_constant__ Sources s) {
    begin_and_let_next_begin();
    wait_for_earlier_kernels();
    const int which = blockIdx.y;
    const auto &sh = s.shapes[s.shape[which]];
    const int row0 = static_cast<int>(blockIdx.x) * sh.block_rows;
    if (row0 >= sh.rows) return;
    const int parts = (sh.rows + sh.block_rows - 1) / sh.block_rows, cols = sh.cols, ld = sh.ld;
    double sum = 0;
    for (int i = threadIdx.x; i < parts; i += ORTH_THREADS) sum += s.partial[static_cast<long long>(which) * s.most + i];
    const float factor = static_cast<float>(static_cast<double>(ORTH_UNIT) / (sqrt(block_sum(sum)) + static_cast<double>(s.eps)));
    const long long to = (static_cast<long long>(s.number[which]) * sh.rows + row0) * ld;
    __half *const hi = sh.hi + to, *const lo = sh.lo + to;
    visit<UT, GT>(s, which, static_cast<long long>(row0) * cols, min(sh.block_rows, sh.rows - row0) * cols, [&](int i, const auto &v) {
        constexpr int N = sizeof(v) / sizeof(float);
        const int r = i / cols;
        const long long at = static_cast<long long>(r) * (ld - cols) + i;
        if constexpr (N == 8) {
            uint32_t h[4], l[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float a = v[2 * e] * factor, b = v[2 * e + 1] * factor;
                h[e] = pack_f16(a, b);
                const float2 x = unpack_f16(h[e]);
                l[e] = pack_f16((a - x.x) * ORTH_LO, (b - x.y) * ORTH_LO);
            }
            *reinterpret_cast<uint4 *>(hi + at) = make_uint4(h[0], h[1], h[2], h[3]);
            *reinterpret_cast<uint4 *>(lo + at) = make_uint4(l[0], l[1], l[2], l[3]);
        } else {
            const float x = v[0] * factor;
            const __half h = __float2half_rn(x);
            hi[at] = h;
            lo[at] = __float2half_rn((x - __half2float(h)) * ORTH_LO);
        }
    });
}

// ---- the products' epilogues -------------------------------------------------------------------------
// Bound: bringing operands and emptying accumulators, nearly alike: 840 matrices of 192 .. 1536 x 576, k as G's is the longer side and of G^2 the shorter one, 4.1 ms of ten such products each
// (1.75 TFLOP, half of them counted).
// A symmetric result: alpha times the sums, plus b times in[0], plus `diagonal` there; pieces below the diagonal go to the other one's place, too.
struct SymEpilogue {
    static constexpr int STAGING = 2048;
    static constexpr bool READS_BOXES = false, WRITES_BOXES = false;   // (as boxes, which the turned ones can be, too, 15 % slower: the copy engine has the operands to bring)
    __device__ static bool wants(const GemmGroup &g, int row0, int col0) { return row0 < g.m && col0 <= row0; }
    float b, diagonal;
    struct Ahead {
        uint4 v[4];
    };
    using Args = GemmArgs<SymEpilogue>;
    __device__ static void fetch(const Args &, const GemmGroup &g, int batch, int row0, int col0, int lane, Ahead &x) {
        if (g.in[0])
            fetch16(static_cast<const __half *>(g.in[0]) + batch * g.out_batch + row0 * g.out_ld + col0, g.out_ld, piece_at(g, row0, col0, true), lane, x.v);
    }
    __device__ static void settle(const Args &, const GemmGroup &g, int, int row0, int col0, char *st, int lane, const Ahead &x) {
        settle16(st, lane, nullptr, 0, piece_at(g, row0, col0, true), x.v);
    }
    __device__ static void drain(const Args &a, const GemmGroup &g, int batch, int row0, int col0, uint32_t d, char *st, const char *, int lane) {
        const Piece p = piece_at(g, row0, col0, true);
        __half *const out = static_cast<__half *>(g.out[0]) + batch * g.out_batch;
        // Columns of a piece below the diagonal are rows of the other one (p.cols is 32 there).  Neighbouring lanes, neighbouring rows of this piece, make words: the even
        // one of the even column, the odd one of the odd column.
        const bool odd = lane & 1, both = (lane | 1) < p.rows, one = (lane & ~1) < p.rows;
        uint32_t *t = reinterpret_cast<uint32_t *>(out + (col0 + odd) * g.out_ld + row0 + (lane & ~1));
        float sums[2][16];
        tmem_load16(d, sums[0]);
        tmem_load16(d + 16, sums[1]);
        tmem_wait();
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            float (&v)[16] = sums[half];
            uint32_t w[8];
            if (g.in[0]) row16(st, lane, half, w);
#pragma unroll
            for (int e = 0; e < 16; ++e) v[e] *= g.alpha;
            if (g.in[0]) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float2 x = unpack_f16(w[e]);
                    v[2 * e] += a.epi.b * x.x, v[2 * e + 1] += a.epi.b * x.y;
                }
                if (col0 == row0) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) v[e] += e + 16 * half == lane ? a.epi.diagonal : 0.f;
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = pack_f16(v[2 * e], v[2 * e + 1]);
            put16(st, lane, half, w);
            if (col0 < row0) {
#pragma unroll
                for (int e = 0; e < 8; ++e, t += g.out_ld) {   // (two columns on: 2 ld halves)
                    const uint32_t other = __shfl_xor_sync(0xffffffffu, w[e], 1);
                    const uint32_t pair = odd ? __byte_perm(other, w[e], 0x7632) : __byte_perm(w[e], other, 0x5410);
                    if (both) *t = pair;
                    else if (one) *reinterpret_cast<unsigned short *>(t) = static_cast<unsigned short>(pair);
                }
            }
        }
    }
    __device__ static void send(const Args &, const GemmGroup &g, int batch, int row0, int col0, const char *st, int lane) {
        send16(st, lane, static_cast<__half *>(g.out[0]) + batch * g.out_batch + row0 * g.out_ld + col0, g.out_ld, piece_at(g, row0, col0, true));
    }
};

// X of the next step: alpha times the sums (with a X's larger part in them) and `lo` times its smaller part; in two halves.
// Bound: as above; the same 840 matrices 3.15 ms of four such products each (2.4 TFLOP), 3.3 without boxes.
struct NextEpilogue {
    static constexpr int STAGING = 3 * 2048;
    static constexpr bool READS_BOXES = true, WRITES_BOXES = true;
    float lo;
    int both;   // the smaller part is written, too
    struct Ahead {};
    using Args = GemmArgs<NextEpilogue>;
    __device__ static bool wants(const GemmGroup &g, int row0, int col0) { return row0 < g.m && col0 < g.n; }
    __device__ static void drain(const Args &a, const GemmGroup &g, int, int, int, uint32_t d, char *st, const char *input, int lane) {
        float sums[2][16];
        tmem_load16(d, sums[0]);
        tmem_load16(d + 16, sums[1]);
        tmem_wait();
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            float (&v)[16] = sums[half];
            uint32_t hi[8], lo[8];
            row16(input, lane, half, lo);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float2 l = unpack_f16(lo[e]);
                v[2 * e] = v[2 * e] * g.alpha + a.epi.lo * l.x, v[2 * e + 1] = v[2 * e + 1] * g.alpha + a.epi.lo * l.y;
                hi[e] = pack_f16(v[2 * e], v[2 * e + 1]);
                const float2 h = unpack_f16(hi[e]);
                lo[e] = pack_f16((v[2 * e] - h.x) * ORTH_LO, (v[2 * e + 1] - h.y) * ORTH_LO);
            }
            if (a.epi.both) put16(const_cast<char *>(input), lane, half, lo);
            put16(st + 4096, lane, half, hi);
        }
    }
    __device__ static void send_boxes(const Args &a, const GemmGroup &g, int batch, int row0, int col0, const char *st, const char *input) {
        tma_store(&a.maps[g.out_map], col0, row0, g.io_batch + batch, st + 4096);
        if (a.epi.both) tma_store(&a.maps[g.in_map], col0, row0, g.io_batch + batch, input);
    }
    __device__ static void send(const Args &, const GemmGroup &, int, int, int, const char *, int) {}
};

// What the last step gives: to a tensor of the caller's, or into the step of x.  (The smaller part of X has no place in it: no step follows that would enlarge what is rounded
// away here, 2^-12 of X times a.)
enum { ORTH_TO_F32 = 0, ORTH_TO_BF16 = 1, ORTH_TO_X = 2 };
template <int TO>
struct LastEpilogue {
    static constexpr int STAGING = TO == ORTH_TO_BF16 ? 2048 : 4096;
    static constexpr bool READS_BOXES = false, WRITES_BOXES = false;
    __device__ static bool wants(const GemmGroup &g, int row0, int col0) { return row0 < g.m && col0 < g.n; }
    float scale[ORTH_SHAPES];         // of the shape: with 1 / ORTH_UNIT^2; of the step with the learning rate
    float decay;
    void *out[ORTH_ROUND];
    float *const *table;
    int index[ORTH_ROUND];
    struct Ahead {
        uint4 x[TO == ORTH_TO_X ? 8 : 1];
    };
    using Args = GemmArgs<LastEpilogue>;
    __device__ __forceinline__ static void *to(const Args &a, const GemmGroup &g, int batch) {
        if constexpr (TO == ORTH_TO_X) return a.epi.table[a.epi.index[g.first + batch]];
        else return a.epi.out[g.first + batch];
    }
    __device__ __forceinline__ static Piece piece(const GemmGroup &g, const void *out, int row0, int col0) {
        constexpr int SIZE = TO == ORTH_TO_BF16 ? 2 : 4;
        return piece_at(g, row0, col0, ((reinterpret_cast<uintptr_t>(out) | static_cast<uintptr_t>(g.out_ld * SIZE)) & 15) == 0);
    }
    __device__ static void fetch(const Args &a, const GemmGroup &g, int batch, int row0, int col0, int lane, Ahead &x) {
        if constexpr (TO == ORTH_TO_X) {
            const float *out = static_cast<const float *>(to(a, g, batch));
            fetch32(out + row0 * g.out_ld + col0, g.out_ld, piece(g, out, row0, col0), lane, x.x);
        }
    }
    __device__ static void settle(const Args &, const GemmGroup &, int, int, int, char *st, int lane, const Ahead &x) {
        if constexpr (TO == ORTH_TO_X) settle32(st, lane, x.x);
    }
    __device__ static void drain(const Args &a, const GemmGroup &g, int batch, int row0, int col0, uint32_t d, char *st, const char *, int lane) {
        const float scale = a.epi.scale[&g - a.groups];
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {
            float v[16];
            tmem_load16(d + 16 * half, v);
            tmem_wait();
            if constexpr (TO == ORTH_TO_BF16) {
                uint32_t w[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = pack_bf16(v[2 * e] * scale, v[2 * e + 1] * scale);
                put16(st, lane, half, w);
            } else {
                if constexpr (TO == ORTH_TO_X) {
                    float x[16];
                    row32(st, lane, half, x);
#pragma unroll
                    for (int e = 0; e < 16; ++e) v[e] = a.epi.decay * x[e] - scale * v[e];
                } else {
#pragma unroll
                    for (int e = 0; e < 16; ++e) v[e] *= scale;
                }
                put32(st, lane, half, v);
            }
        }
    }
    __device__ static void send(const Args &a, const GemmGroup &g, int batch, int row0, int col0, const char *st, int lane) {
        void *const out = to(a, g, batch);
        const Piece p = piece(g, out, row0, col0);
        const long long at = row0 * g.out_ld + col0;
        if constexpr (TO == ORTH_TO_BF16) send16(st, lane, static_cast<__nv_bfloat16 *>(out) + at, g.out_ld, p);
        else send32(st, lane, static_cast<float *>(out) + at, g.out_ld, p);
    }
};

// ---- rounds ------------------------------------------------------------------------------------------
int64_t padded(int64_t n) { return (n + 7) & ~int64_t{7}; }

struct Shape {
    int rows, cols, count, first;     // matrices [first, first + count) of the round
    int n, m;                         // the shorter and the longer side
    bool tall;
    int64_t ld, square_ld;
    __half *hi[2], *lo, *gram, *poly;
};
struct Round {
    int first, count;                 // of the sorted list
    int nshapes;
    Shape shapes[ORTH_SHAPES];
    int64_t bytes;
};
int64_t matrix_bytes(int rows, int cols) {
    const int64_t n = std::min(rows, cols);
    return 6 * rows * padded(cols) + 4 * n * padded(n);
}
int block_rows(int cols) { return std::max(ORTH_WARPS, (16384 / std::max(cols, 1)) / ORTH_WARPS * ORTH_WARPS); }

// The matrices from `first` on that are taken at once.  The more, the better the SMs' rounds of tiles are filled and the fewer launches wait for the ones in front of them
// (840 matrices of a 135 M-parameter model and its replicas: 12.1 ms of 128 at a time, 14.9 ms of so few that L2 holds them): up to ORTH_ROUND_BYTES of working memory,
// the rounds alike.
constexpr int64_t ORTH_ROUND_BYTES = 2ll << 30;
Round next_round(const OrthArgs &a, int first) {
    int64_t rest = 0;
    for (int i = first; i < a.count; ++i) rest += matrix_bytes(a.list[i].rows, a.list[i].cols);
    const int64_t rounds = std::max((rest + ORTH_ROUND_BYTES - 1) / ORTH_ROUND_BYTES, static_cast<int64_t>((a.count - first + ORTH_ROUND - 1) / ORTH_ROUND));
    const int64_t fair = rest / rounds;
    Round r{};
    r.first = first;
    while (first + r.count < a.count && r.count < ORTH_ROUND) {
        const OrthMatrix &x = a.list[first + r.count];
        const int64_t bytes = matrix_bytes(x.rows, x.cols);
        if (r.count > 0 && rounds > 1 && r.bytes + bytes / 2 > fair) break;
        if (r.nshapes == 0 || r.shapes[r.nshapes - 1].rows != x.rows || r.shapes[r.nshapes - 1].cols != x.cols) {
            if (r.nshapes == ORTH_SHAPES) break;
            Shape &s = r.shapes[r.nshapes++];
            s.rows = x.rows, s.cols = x.cols, s.count = 0, s.first = r.count;
            s.n = std::min(x.rows, x.cols), s.m = std::max(x.rows, x.cols), s.tall = x.rows > x.cols;
            s.ld = padded(x.cols), s.square_ld = padded(s.n);
        }
        ++r.shapes[r.nshapes - 1].count;
        ++r.count;
        r.bytes += bytes;
    }
    return r;
}
// Places everything of a round in working memory; its end.
int64_t place(Round &r, char *work, double **partial, int *most) {
    int64_t used = 0;
    const auto take = [&](int64_t bytes) {
        char *p = work ? work + used : nullptr;
        used += (bytes + 255) & ~int64_t{255};
        return p;
    };
    int blocks = 1;
    for (int i = 0; i < r.nshapes; ++i) {
        Shape &s = r.shapes[i];
        const int64_t x = s.count * s.rows * s.ld * 2, g = s.count * s.n * s.square_ld * 2;
        for (__half **p : {&s.hi[0], &s.hi[1], &s.lo}) *p = reinterpret_cast<__half *>(take(x));
        s.gram = reinterpret_cast<__half *>(take(g)), s.poly = reinterpret_cast<__half *>(take(g));
        blocks = std::max(blocks, (s.rows + block_rows(s.cols) - 1) / block_rows(s.cols));
    }
    double *const p = reinterpret_cast<double *>(take(static_cast<int64_t>(r.count) * blocks * 8));
    if (partial) *partial = p, *most = blocks;
    return used;
}

// Small matrices first, then by shape; how many small ones.
int sort_list(const OrthArgs &a) {
    std::sort(a.list, a.list + a.count, [](const OrthMatrix &x, const OrthMatrix &y) {
        const bool sx = orth_is_small(x.rows, x.cols), sy = orth_is_small(y.rows, y.cols);
        return sx != sy ? sx : x.rows != y.rows ? x.rows < y.rows : x.cols != y.cols ? x.cols < y.cols : x.index < y.index;
    });
    int small = 0;
    while (small < a.count && orth_is_small(a.list[small].rows, a.list[small].cols)) ++small;
    return small;
}

// What the result is multiplied by.
double scale_of(const OrthArgs &a, int rows, int cols) {
    const double scale = a.scale == DESLOC_SCALE_ASPECT ? std::sqrt(std::max(1.0, static_cast<double>(rows) / cols))
                         : a.scale == DESLOC_SCALE_RMS  ? 0.2 * std::sqrt(static_cast<double>(std::max(rows, cols)))
                                                        : 1.0;
    return scale * (a.list[0].out ? 1.0 : static_cast<double>(a.lr));
}

// The cut of a product of all shapes: tiles(shape, cut) of one matrix, k(shape).
template <typename K, typename F>
GemmCut pick(const Round &r, bool symmetric, const K &k, const F &tiles) {
    int64_t all = 0, sum = 0;
    for (int i = 0; i < r.nshapes; ++i) {
        const int64_t n = static_cast<int64_t>(r.shapes[i].count) * tiles(r.shapes[i], GemmCut{256, true});
        all += n, sum += n * k(r.shapes[i]);
    }
    return pick_cut(false, GEMM_BM, sum / all, [&](const GemmCut &cut) {
        TileCount n{0, 0};
        const int rows = GEMM_BM * (cut.pairs ? 2 : 1);
        for (int i = 0; i < r.nshapes; ++i) {
            const Shape &s = r.shapes[i];
            n.all += static_cast<int64_t>(s.count) * tiles(s, cut);
            if (symmetric && cut.tile_n == rows) n.once += static_cast<int64_t>(s.count) * ((s.n + rows - 1) / rows);
        }
        return n;
    });
}

struct Run {
    cudaStream_t stream;
    int *err, wait_limit, *launches;
};

// A symmetric product of `from` (x: X of this step, else G) for all shapes.
cudaError_t symmetric(const Round &r, bool gram, int side, float alpha, float b, float diagonal, const Run &run) {
    static thread_local GemmArgs<SymEpilogue> a;
    const GemmCut cut = pick(r, true, [&](const Shape &s) { return gram ? s.m : s.n; }, [](const Shape &s, const GemmCut &c) { return tiles_of(s.n, s.n, c, false, true); });
    begin_gemm(a, false, cut, false, true, 1);
    a.epi.b = b, a.epi.diagonal = diagonal;
    for (int i = 0; i < r.nshapes; ++i) {
        const Shape &s = r.shapes[i];
        const bool mn = gram && s.tall;
        GemmGroup &g = add_group(a, s.n, s.n, gram ? s.m : s.n, s.count);
        for (int side_b = 0; side_b < 2; ++side_b) {
            const int box = mn ? 64 : side_b ? cut.box_n(false) : box_rows(s.n);
            const cudaError_t e = gram ? encode_boxes(&a.maps[2 * i + side_b], s.hi[side], false, s.cols, s.rows, s.count, s.ld, s.rows * s.ld, box)
                                       : encode_boxes(&a.maps[2 * i + side_b], s.gram, false, s.n, s.n, s.count, s.square_ld, s.n * s.square_ld, box);
            if (e != cudaSuccess) return e;
        }
        g.a_map = static_cast<short>(2 * i), g.b_map = static_cast<short>(2 * i + 1);
        g.a_mn = g.b_mn = mn;
        g.alpha = alpha;
        g.out[0] = gram ? s.gram : s.poly;
        g.in[0] = gram ? nullptr : s.gram;
        g.out_ld = s.square_ld, g.out_batch = s.n * s.square_ld;
    }
    return launch_gemm(a, run.err, run.wait_limit, run.stream, run.launches);
}

// X := a X + (polynomial of G) X, to the other side or, at last, to `epi`'s places.
template <typename E>
cudaError_t update(const Round &r, int side, const E &epi, GemmArgs<E> &a, const long long *out_ld, const Run &run) {
    const GemmCut cut = pick(r, false, [](const Shape &s) { return s.n; }, [](const Shape &s, const GemmCut &c) { return tiles_of(s.rows, s.cols, c, false, false); });
    begin_gemm(a, false, cut, false, false, 1);
    a.epi = epi;
    for (int i = 0; i < r.nshapes; ++i) {
        const Shape &s = r.shapes[i];
        GemmGroup &g = add_group(a, s.rows, s.cols, s.n, s.count);
        const int of_x = 2 * i + (s.tall ? 0 : 1), of_poly = 2 * i + (s.tall ? 1 : 0);
        cudaError_t e = encode_boxes(&a.maps[of_x], s.hi[side], false, s.cols, s.rows, s.count, s.ld, s.rows * s.ld, s.tall ? box_rows(s.rows) : 64);
        if (e == cudaSuccess)
            e = encode_boxes(&a.maps[of_poly], s.poly, false, s.n, s.n, s.count, s.square_ld, s.n * s.square_ld, s.tall ? cut.box_n(false) : box_rows(s.n));
        if (!out_ld) {
            const int boxes = 2 * ORTH_SHAPES + 2 * i;
            if (e == cudaSuccess) e = encode_boxes(&a.maps[boxes], s.hi[side ^ 1], false, s.cols, s.rows, s.count, s.ld, s.rows * s.ld, 32, 32);
            if (e == cudaSuccess) e = encode_boxes(&a.maps[boxes + 1], s.lo, false, s.cols, s.rows, s.count, s.ld, s.rows * s.ld, 32, 32);
            g.out_map = static_cast<short>(boxes), g.in_map = static_cast<short>(boxes + 1);
        }
        if (e != cudaSuccess) return e;
        g.a_map = static_cast<short>(2 * i), g.b_map = static_cast<short>(2 * i + 1);
        g.b_mn = !s.tall;
        g.alpha = 1.f / ORTH_UNIT;
        g.out_ld = out_ld ? out_ld[i] : s.ld;
        g.first = s.first;
    }
    return launch_gemm(a, run.err, run.wait_limit, run.stream, run.launches);
}

template <int TO>
cudaError_t last(const OrthArgs &a, const Round &r, int side, const Run &run) {
    using E = LastEpilogue<TO>;
    static thread_local GemmArgs<E> args;
    static thread_local E epi;
    epi.decay = a.decay;
    epi.table = a.x_table;
    long long ld[ORTH_SHAPES];
    for (int i = 0; i < r.nshapes; ++i) {
        const Shape &s = r.shapes[i];
        epi.scale[i] = a.list[r.first + s.first].scale / (ORTH_UNIT * ORTH_UNIT);
        ld[i] = s.cols;
    }
    for (int i = 0; i < r.count; ++i) epi.out[i] = a.list[r.first + i].out, epi.index[i] = a.list[r.first + i].index;
    return update(r, side, epi, args, ld, run);
}

template <typename UT, typename GT>
cudaError_t prepare(const Sources &s, int count, const Run &run) {
    const dim3 grid(s.most, count);
    cudaError_t e = launch_op(orth_norm_kernel<UT, GT>, grid, dim3(ORTH_THREADS), 0, true, run.stream, s);
    if (e == cudaSuccess) ++*run.launches, e = launch_op(orth_scale_kernel<UT, GT>, grid, dim3(ORTH_THREADS), 0, true, run.stream, s);
    if (e == cudaSuccess) ++*run.launches;
    return e;
}

}  // namespace

int64_t orth_work(const OrthArgs &a) {
    int64_t most = 256;
    for (int at = sort_list(a); at < a.count;) {
        Round r = next_round(a, at);
        most = std::max(most, place(r, nullptr, nullptr, nullptr));
        at += r.count;
    }
    return most;
}

cudaError_t launch_orth(const OrthArgs &a, char *work, int *err, int wait_limit, cudaStream_t stream, int *launches) {
    const Run run{stream, err, wait_limit, launches};
    const int small = sort_list(a);
    for (int i = 0; i < a.count; ++i) a.list[i].scale = static_cast<float>(scale_of(a, a.list[i].rows, a.list[i].cols));
    if (small > 0) {
        const cudaError_t e = launch_orth_small(a, 0, small, err, wait_limit, stream, launches);
        if (e != cudaSuccess) return e;
    }
    static thread_local Sources s;
    static thread_local GemmArgs<NextEpilogue> next;
    for (int at = small; at < a.count;) {
        Round r = next_round(a, at);
        place(r, work, &s.partial, &s.most);
        s.table = a.u_table, s.beta = a.beta, s.eps = a.eps, s.rho = a.rho;
        for (int i = 0; i < r.nshapes; ++i) {
            const Shape &sh = r.shapes[i];
            s.shapes[i] = {sh.rows, sh.cols, static_cast<int>(sh.ld), block_rows(sh.cols), sh.hi[0], sh.lo};
            for (int k = 0; k < sh.count; ++k) {
                const OrthMatrix &x = a.list[at + sh.first + k];
                s.update[sh.first + k] = x.update, s.grad[sh.first + k] = x.grad, s.index[sh.first + k] = x.index;
                s.shape[sh.first + k] = i, s.number[sh.first + k] = k;
            }
        }
        using bf = __nv_bfloat16;
        cudaError_t e = a.update_bf16 ? (a.grad_bf16 ? prepare<bf, bf> : prepare<bf, float>)(s, r.count, run)
                                      : (a.grad_bf16 ? prepare<float, bf> : prepare<float, float>)(s, r.count, run);
        int side = 0;
        for (int k = 0; k < a.steps && e == cudaSuccess; ++k, side ^= 1) {
            const float *c = a.coefficients + 3 * k;
            e = symmetric(r, true, side, 1.f / ORTH_UNIT, 0.f, 0.f, run);
            if (e == cudaSuccess) e = symmetric(r, false, side, c[2] / ORTH_UNIT, c[1], c[0] * ORTH_UNIT, run);
            if (e != cudaSuccess) break;
            if (k + 1 < a.steps) e = update(r, side, NextEpilogue{c[0] / ORTH_LO, k + 2 < a.steps}, next, nullptr, run);
            else if (a.list[at].out == nullptr) e = last<ORTH_TO_X>(a, r, side, run);
            else e = a.out_bf16 ? last<ORTH_TO_BF16>(a, r, side, run) : last<ORTH_TO_F32>(a, r, side, run);
        }
        if (e != cudaSuccess) return e;
        at += r.count;
    }
    return cudaSuccess;
}

}  // namespace desloc
