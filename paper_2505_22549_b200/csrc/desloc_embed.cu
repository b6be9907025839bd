// Embedding lookup from the workers' replicas, and its gradient by sorted tokens.
#include "desloc_ops.cuh"

#include <type_traits>

namespace desloc {

namespace {

// ---- lookup ------------------------------------------------------------------------------------------
// out[m, i, :] = scale * x^m[token(m, i), :].  Bound: HBM, 4 bytes read (rows that occur again come from L2) and 2 or 4 written per
// element.  `blockDim.x` lanes take a row, four 16-byte loads in flight each.  4 workers x 8192 tokens, width 2048, to bf16: 42.4 us, 6.0 TB/s (0.92 of
// copy); with 64 and 128 lanes a row 42.2 and 45.6, with registers for twice the blocks 59.7.  One token per worker: 2.6 us, the launch and three
// dependent loads.
constexpr int EMBED_THREADS = 128;

// N columns at a time, four times as many in flight.
template <int N, typename OT>
__device__ __forceinline__ void embed_row(const float *row, OT *out, int width, float scale, bool none) {
    const int lanes = blockDim.x, n = width / N;
    for (int c = threadIdx.x; c < n; c += 4 * lanes) {
        float f[4][N];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (!none && c + k * lanes < n) load_values(row + N * (c + k * lanes), f[k]);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (c + k * lanes >= n) break;
#pragma unroll
            for (int e = 0; e < N; ++e) f[k][e] = none ? 0.f : f[k][e] * scale;
            store_values(out + N * (c + k * lanes), f[k]);
        }
    }
}

template <typename OT>
__global__ void __launch_bounds__(EMBED_THREADS) embed_kernel(const EmbedArgs a) {
    begin_and_let_next_begin();
    const int m = blockIdx.y, i = static_cast<int>(blockIdx.x * blockDim.y + threadIdx.y);
    wait_for_earlier_kernels();
    if (i >= a.n) return;
    const int tok = token_at(a.tokens, m * a.tokens.s0 + i * a.tokens.s1, a.vocab);
    OT *out = static_cast<OT *>(a.out) + m * a.os0 + i * a.os1;
    const float *row = a.x[static_cast<long long>(m) * a.x_stride] + static_cast<long long>(max(tok, 0)) * a.width;
    const auto on = [&](unsigned n) {
        return a.width % n == 0 && reinterpret_cast<uintptr_t>(row) % (4 * n) == 0 && reinterpret_cast<uintptr_t>(out) % (n * sizeof(OT)) == 0;
    };
    if (on(4)) embed_row<4>(row, out, a.width, a.scale, tok < 0);
    else if (on(2)) embed_row<2>(row, out, a.width, a.scale, tok < 0);
    else embed_row<1>(row, out, a.width, a.scale, tok < 0);
}

// ---- sort --------------------------------------------------------------------------------------------
// Stable counting sort of a worker's tokens, a block for each value of the tokens' last bits: it goes over all of them twice, counts
// its own and those of the blocks in front of it, and writes its places.  A run is the places of one token.  No block waits for another.
// Bound: latency; up to SORT_CACHED tokens stay in registers between the two times.  4 x 8192 tokens of 49152: 17 us alone, in which the blocks behind
// it write zeros.  (Blocks of 512 threads 18 us; all 8192 tokens in registers 15 us, but the zeros then have two blocks per SM instead of three: 78 us
// in all instead of 70.)
constexpr int SORT_THREADS = 256, SORT_WARPS = SORT_THREADS / 32, SORT_AHEAD = 16;
constexpr int SORT_CACHED = SORT_THREADS * SORT_AHEAD;
constexpr int SORT_KEYS = 768;   // most numbers that a block tells apart: 30 KB of shared memory

// A run of `piece` or more places is cut into floor(length / piece) pieces of nearly equal length, summed by a block each.  Piece j of
// a run that begins at place s has number ceil(s / piece) + j: no two runs' numbers meet, because ceil(a + b) >= ceil(a) + floor(b), and
// place number * piece lies in the run.
struct Pieces {
    int first, n;
    __device__ __forceinline__ Pieces(const EmbedGradArgs &a, int start, int length)
        : first((start + a.piece - 1) / a.piece), n(length / a.piece) {}
};

// Zeros over `bytes` bytes (a multiple of two) from p on, by a warp.
__device__ __forceinline__ void zero_span(char *p, long long bytes) {
    const int lane = threadIdx.x & 31;
    const int head = static_cast<int>(min(bytes, static_cast<long long>((0 - reinterpret_cast<uintptr_t>(p)) & 15u)));
    const long long wide = (bytes - head) / 16;
    const int rest = static_cast<int>(bytes - head - 16 * wide);
    if (2 * lane < head) *reinterpret_cast<unsigned short *>(p + 2 * lane) = 0;
    uint4 *w = reinterpret_cast<uint4 *>(p + head);
#pragma unroll 4
    for (long long i = lane; i < wide; i += 32) w[i] = make_uint4(0, 0, 0, 0);
    if (2 * lane < rest) *reinterpret_cast<unsigned short *>(p + head + 16 * wide + 2 * lane) = 0;
}

// Zeros in the rows [v0, v0 + rows) that have no bit in `seen`, `each` of them (at most 32) per warp,
// neighbouring ones at once.
template <typename GT>
__device__ __forceinline__ void zero_rows(const EmbedGradArgs &a, int m, int v0, int each, unsigned seen) {
    unsigned long long todo = ~static_cast<unsigned long long>(seen) & ((1ull << min(each, max(a.vocab - v0, 0))) - 1);
    GT *const out = static_cast<GT *>(a.g[m]);
    while (todo) {
        const int r = __ffsll(static_cast<long long>(todo)) - 1, n = __ffsll(static_cast<long long>(~(todo >> r))) - 1;
        zero_span(reinterpret_cast<char *>(out + static_cast<long long>(v0 + r) * a.width), n * (static_cast<long long>(a.width) * sizeof(GT)));
        todo &= ~(((1ull << n) - 1) << r);
    }
}

// The rows [block * zero_rows, ...) of the gradient that no token of the worker's stands for: zeros.
constexpr int ZERO_ROWS = 32, MOST_ZERO_ROWS = 16 * SORT_WARPS, ZERO_BYTES = 300 * 1024, ZEROS_AHEAD = 16384;   // (a block goes over all tokens: 2 us for 8192)

template <bool WIDE, typename GT>
__device__ __forceinline__ void zero_block(const EmbedGradArgs &a, int m, unsigned block, int rows) {
    using Number = std::conditional_t<WIDE, long long, int>;
    __shared__ unsigned s_seen[MOST_ZERO_ROWS / 32];
    const int tid = threadIdx.x, warp = tid >> 5, v0 = static_cast<int>(block) * rows, each = rows / SORT_WARPS;
    if (tid < MOST_ZERO_ROWS / 32) s_seen[tid] = 0;
    __syncthreads();
    wait_for_earlier_kernels();
    const Number *const tokens = static_cast<const Number *>(a.tokens.data) + m * a.tokens.s0;
#pragma unroll 8
    for (int i = tid; i < a.n; i += SORT_THREADS) {
        using Unsigned = std::make_unsigned_t<Number>;
        const Unsigned r = static_cast<Unsigned>(tokens[i * a.tokens.s1]) - static_cast<Unsigned>(v0);
        if (r < static_cast<unsigned>(rows)) atomicOr(&s_seen[r / 32], 1u << (r % 32));
    }
    __syncthreads();
    zero_rows<GT>(a, m, v0 + warp * each, each, s_seen[warp * each / 32] >> (warp * each % 32));
}

// WIDE: 64-bit token numbers.  Behind the sort's own blocks, `zero_blocks` per worker that write the gradient's zeros meanwhile.
template <bool CACHED, bool WIDE, typename GT>
__global__ void __launch_bounds__(SORT_THREADS, 3) token_sort_kernel(const __grid_constant__ EmbedGradArgs a, int M, unsigned zero_blocks, int rows) {
    using Number = std::conditional_t<WIDE, long long, int>;
    extern __shared__ int hist[];   // [warp][key]: counts, then places; then [key] first place and length
    __shared__ int s_warp[SORT_WARPS];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const unsigned sort_blocks = static_cast<unsigned>(M) << a.bits;
    if (blockIdx.x >= sort_blocks) {
        begin_and_let_next_begin();
        const unsigned block = blockIdx.x - sort_blocks, m = block / zero_blocks;
        return zero_block<WIDE, GT>(a, static_cast<int>(m), block - m * zero_blocks, rows);
    }
    const int mask = (1 << a.bits) - 1, b = static_cast<int>(blockIdx.x) & mask, m = static_cast<int>(blockIdx.x >> a.bits);
    int *const mine = hist + warp * a.keys, *const run_start = hist + SORT_WARPS * a.keys, *const run_length = run_start + a.keys;
    begin_and_let_next_begin();
    for (int k = tid; k < SORT_WARPS * a.keys; k += SORT_THREADS) hist[k] = 0;
    __syncthreads();
    wait_for_earlier_kernels();
    // a warp's share: consecutive positions, so that places by (key, warp) are places by (key, position)
    const int share = (a.n + SORT_THREADS - 1) / SORT_THREADS * 32;
    const int lo = static_cast<int>(min(static_cast<long long>(a.n), static_cast<long long>(warp) * share)), hi = min(a.n - lo, share) + lo;
    const Number *const tokens = static_cast<const Number *>(a.tokens.data) + m * a.tokens.s0;
    int t[SORT_AHEAD];
    const auto load = [&](int i0) {
        const Number *p = tokens + (i0 + lane) * a.tokens.s1;
        const long long step = 32 * a.tokens.s1;
        Number v[SORT_AHEAD];
#pragma unroll
        for (int k = 0; k < SORT_AHEAD; ++k) v[k] = i0 + 32 * k < hi - lane ? p[k * step] : -1;
#pragma unroll
        for (int k = 0; k < SORT_AHEAD; ++k)
            t[k] = static_cast<std::make_unsigned_t<Number>>(v[k]) < static_cast<unsigned>(a.vocab) ? static_cast<int>(v[k]) : -1;
    };
    int before = 0;
    for (int i0 = lo; i0 < hi; i0 += 32 * SORT_AHEAD) {
        load(i0);
#pragma unroll
        for (int k = 0; k < SORT_AHEAD; ++k) {
            const int last = t[k] < 0 ? mask + 1 : t[k] & mask;
            if (last == b) atomicAdd(&mine[t[k] >> a.bits], 1);
            before += last < b;
        }
    }
    before = __reduce_add_sync(0xffffffffu, before);
    if (lane == 0) s_warp[warp] = before;
    __syncthreads();
    int base = 0;
#pragma unroll
    for (int w = 0; w < SORT_WARPS; ++w) base += s_warp[w];
    // places: keys in order, the warps of a key in order
    for (int k0 = 0; k0 < a.keys; k0 += SORT_THREADS) {
        const int key = k0 + tid;
        int total = 0;
        if (key < a.keys)
#pragma unroll
            for (int w = 0; w < SORT_WARPS; ++w) total += hist[w * a.keys + key];
        int upto = total;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int o = __shfl_up_sync(0xffffffffu, upto, off);
            if (lane >= off) upto += o;
        }
        __syncthreads();   // s_warp has been read
        if (lane == 31) s_warp[warp] = upto;
        __syncthreads();
        int front = 0, all = 0;
#pragma unroll
        for (int w = 0; w < SORT_WARPS; ++w) {
            front += w < warp ? s_warp[w] : 0;
            all += s_warp[w];
        }
        int at = base + front + upto - total;
        const long long v = (static_cast<long long>(key) << a.bits) | b;
        if (key < a.keys && v < a.vocab) {
            a.seen[static_cast<long long>(m) * a.vocab + v] = total > 0;
            if (total > 0) {
                run_start[key] = at;
                run_length[key] = total;
                if (total >= a.piece) {
                    const long long ticket = static_cast<long long>(m) * a.pieces + Pieces(a, at, total).first;
                    for (int c = 0; c < a.columns; ++c) a.tickets[ticket * a.columns + c] = 0;
                }
#pragma unroll
                for (int w = 0; w < SORT_WARPS; ++w) {
                    const int c = hist[w * a.keys + key];
                    hist[w * a.keys + key] = at;
                    at += c;
                }
            }
        }
        base += all;
    }
    if (b == mask && tid == 0) a.count[m] = base;
    __syncthreads();
    int4 *const places = a.places + static_cast<long long>(m) * a.n;
    for (int i0 = lo; i0 < hi; i0 += 32 * SORT_AHEAD) {
        if (!CACHED) load(i0);
#pragma unroll
        for (int k = 0; k < SORT_AHEAD; ++k) {
            const bool is = t[k] >= 0 && (t[k] & mask) == b;
            const unsigned who = __ballot_sync(0xffffffffu, is);
            if (who == 0) continue;
            if (is) {
                const int key = t[k] >> a.bits;
                const unsigned same = __match_any_sync(who, key);
                const int rank = __popc(same & ((1u << lane) - 1));
                const int at = mine[key];
                places[at + rank] = make_int4(i0 + 32 * k + lane, t[k], run_start[key], run_length[key]);
                __syncwarp(who);
                if (rank == 0) mine[key] = at + __popc(same);
            }
            __syncwarp();
        }
    }
}

// ---- sums --------------------------------------------------------------------------------------------
// One launch; a warp takes 32 * N columns of a piece of a long run, or of the short runs that begin in TILE places.  Behind them (where the sort's launch
// has not written them) zeros in the rows without a token, which are most of a large vocabulary.  No barriers: warps wait for their loads alone.
// Bound: HBM, rows of dout read and the gradient written; then the latency of three loads in a row (place, position, row of dout) at 28 warps per SM.
// 4 workers x 8192 tokens, 49152 rows, bf16: width 576 65.5 us in both launches (41 at the copy rate), width 2048 161 (143).  Before, at width 576: a
// block per 16 rows of the gradient 226 us (most blocks wait for one row's loads), the same with zeros and sums by threads 93, tiles of places with pieces
// of long runs by whole blocks 82, pieces by warps 70, blocks of four warps instead of eight 65.5.  Zeros in the sums' warps, behind a sort alone: 65, but
// width 2048 171 and small problems 12 instead of 9.
constexpr int SUM_THREADS = 128, SUM_WARPS = SUM_THREADS / 32;
constexpr int TILE = 8;

// Rows in flight, unpacked when they are added: a row costs four registers.
template <int N, typename ST>
struct RowWords {
    using Word = std::conditional_t<N == 1, ST, std::conditional_t<N == 2, std::conditional_t<sizeof(ST) == 2, uint32_t, uint2>, uint4>>;
    static constexpr int WORDS = N <= 2 ? 1 : N * static_cast<int>(sizeof(ST)) / 16;
    Word w[WORDS];
    __device__ __forceinline__ void load(const ST *p) {
#pragma unroll
        for (int q = 0; q < WORDS; ++q) w[q] = reinterpret_cast<const Word *>(p)[q];
    }
    __device__ __forceinline__ void add_to(float (&acc)[N]) const {
        float f[N];
        load_values(reinterpret_cast<const ST *>(w), f);
#pragma unroll
        for (int e = 0; e < N; ++e) acc[e] += f[e];
    }
};

template <int N, typename GT>
__device__ __forceinline__ void write_sum(const EmbedGradArgs &a, GT *out, const float (&acc)[N]) {
    float v[N] = {};
    if (a.accumulate) load_values(out, v);
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = a.accumulate ? fmaf(acc[e], a.scale, v[e]) : acc[e] * a.scale;
    store_values(out, v);
}

// Adds the rows of dout at places [lo, hi), in order, N columns from `base` on per lane (`in`: there are any), and calls finish(acc, place) with the
// sum behind every place whose bit is set in ends(first place of 32) and starts anew.  The lanes hold the positions of 32 places.
template <int N, typename ST, typename Ends, typename Finish>
__device__ __forceinline__ void add_places(const int4 *places, int n, int lo, int hi, const ST *base, long long stride, bool in, const Ends &ends,
                                           const Finish &finish) {
    constexpr int AHEAD = N * sizeof(ST) > 16 ? 4 : 8;
    const int lane = threadIdx.x & 31;
    float acc[N] = {};
    for (int s0 = lo; s0 < hi; s0 += 32) {
        const int4 q = places[min(s0 + lane, n - 1)];
        const unsigned last = ends(q, s0 + lane);
        const int upto = min(32, hi - s0);
        for (int i0 = 0; i0 < upto; i0 += AHEAD) {
            RowWords<N, ST> row[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
                if (i0 + k < upto) {
                    const int position = __shfl_sync(0xffffffffu, q.x, i0 + k);
                    if (in) row[k].load(base + position * stride);
                }
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
                if (i0 + k < upto) {
                    if (in) row[k].add_to(acc);
                    if (last >> (i0 + k) & 1u) {
                        finish(acc, __shfl_sync(0xffffffffu, q.y, i0 + k));
#pragma unroll
                        for (int e = 0; e < N; ++e) acc[e] = 0.f;
                    }
                }
        }
    }
}

// The short runs that begin in places [s0, s0 + TILE): their places follow one another from the first beginning on; a long run that begins
// here is the last one.
template <typename ST, typename GT, int N>
__device__ __forceinline__ void sum_runs(const EmbedGradArgs &a, int m, int s0, int col) {
    const int lane = threadIdx.x & 31, count = a.count[m];
    const int4 *const places = a.places + static_cast<long long>(m) * a.n;
    const int4 q = places[min(s0 + lane % TILE, a.n - 1)];   // position, token, first place and length of the run (beyond `count`: anything)
    const unsigned begins = __ballot_sync(0xffffffffu, lane < TILE && s0 + lane < count && q.z == s0 + lane);
    if (begins == 0) return;
    const int last = 31 - __clz(begins), length = __shfl_sync(0xffffffffu, q.w, last);
    const bool in = col < a.width;
    GT *const out = static_cast<GT *>(a.g[m]) + col;
    add_places<N>(
        places, a.n, s0 + __ffs(begins) - 1, s0 + last + (length < a.piece ? length : 0), static_cast<const ST *>(a.dout) + m * a.ds0 + col, a.ds1, in,
        [](const int4 &q, int place) { return __ballot_sync(0xffffffffu, place + 1 == q.z + q.w); },
        [&](const float(&acc)[N], int tok) {
            if (in) write_sum<N>(a, out + static_cast<long long>(tok) * a.width, acc);
        });
}

// Piece number p of long runs, if it stands for one.  The last warp of a run's to arrive adds the pieces in their order and writes the row.
template <typename ST, typename GT, int N>
__device__ __forceinline__ void sum_piece(const EmbedGradArgs &a, int m, int p, int c, int col) {
    const int lane = threadIdx.x & 31;
    const long long place = static_cast<long long>(p) * a.piece;
    const int4 *const places = a.places + static_cast<long long>(m) * a.n;
    const int4 q = places[min(place, static_cast<long long>(a.n) - 1)];
    if (place >= a.count[m]) return;
    const Pieces pc(a, q.z, q.w);
    const int j = p - pc.first;
    if (j < 0 || j >= pc.n) return;
    const int lo = q.z + static_cast<int>(static_cast<long long>(q.w) * j / pc.n), hi = q.z + static_cast<int>(static_cast<long long>(q.w) * (j + 1) / pc.n);
    const bool in = col < a.width;
    GT *const out = static_cast<GT *>(a.g[m]) + static_cast<long long>(q.y) * a.width + col;
    float *const part = a.partial + (static_cast<long long>(m) * a.pieces + pc.first) * a.row + col;
    add_places<N>(
        places, a.n, lo, hi, static_cast<const ST *>(a.dout) + m * a.ds0 + col, a.ds1, in,
        [&](const int4 &, int place) { return __ballot_sync(0xffffffffu, place + 1 == hi); },
        [&](const float(&acc)[N], int) {
            if (pc.n == 1) {
                if (in) write_sum<N>(a, out, acc);
            } else if (in) {
                store_values(part + j * a.row, acc);
            }
        });
    if (pc.n == 1) return;
    __threadfence();
    __syncwarp();
    int arrived = 0;
    if (lane == 0) arrived = atomicAdd(&a.tickets[(static_cast<long long>(m) * a.pieces + pc.first) * a.columns + c], 1);
    if (__shfl_sync(0xffffffffu, arrived, 0) != pc.n - 1) return;
    __threadfence();
    if (!in) return;
    float acc[N] = {};
    for (int k0 = 0; k0 < pc.n; k0 += 4) {
        float f[4][N];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k0 + k < pc.n)
#pragma unroll
                for (int e = 0; e < N; e += N <= 2 ? 1 : 4) {
                    if constexpr (N <= 2) {
                        f[k][e] = __ldcg(part + (k0 + k) * a.row + e);
                    } else {
                        const float4 v = __ldcg(reinterpret_cast<const float4 *>(part + (k0 + k) * a.row + e));
                        f[k][e] = v.x, f[k][e + 1] = v.y, f[k][e + 2] = v.z, f[k][e + 3] = v.w;
                    }
                }
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k0 + k < pc.n)
#pragma unroll
                for (int e = 0; e < N; ++e) acc[e] += f[k][e];
    }
    write_sum<N>(a, out, acc);
}

struct SumBlocks {
    unsigned pieces, runs, rows;   // blocks of each kind, per worker
    int block_rows;                // rows that a block of the third kind takes
};

template <typename ST, typename GT, int N>
__global__ void __launch_bounds__(SUM_THREADS, 7) grad_sums_kernel(const __grid_constant__ EmbedGradArgs a, const SumBlocks blocks, int M) {
    begin_and_let_next_begin();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    unsigned block = blockIdx.x;
    wait_for_earlier_kernels();
    // the pieces of all workers first: they take longest
    if (block < (blocks.pieces + blocks.runs) * M) {
        const bool piece = block < blocks.pieces * M;
        if (!piece) block -= blocks.pieces * M;
        const unsigned per = piece ? blocks.pieces : blocks.runs, m = block / per, unit = (block - m * per) * SUM_WARPS + warp, i = unit / a.columns;
        const int c = static_cast<int>(unit - i * a.columns), col = (c * 32 + lane) * N;
        if (piece) return sum_piece<ST, GT, N>(a, static_cast<int>(m), static_cast<int>(i), c, col);
        return sum_runs<ST, GT, N>(a, static_cast<int>(m), static_cast<int>(i) * TILE, col);
    }
    block -= (blocks.pieces + blocks.runs) * M;
    const unsigned m = block / blocks.rows;
    const int each = blocks.block_rows / SUM_WARPS, v0 = static_cast<int>(block - m * blocks.rows) * blocks.block_rows + warp * each;
    const unsigned seen = __ballot_sync(0xffffffffu, lane < each && v0 + lane < a.vocab && a.seen[static_cast<long long>(m) * a.vocab + v0 + lane]);
    zero_rows<GT>(a, static_cast<int>(m), v0, each, seen);
}

template <typename ST, typename GT, int N>
cudaError_t launch_sums(const EmbedGradArgs &a, int M, int64_t zero_blocks, int rows, cudaStream_t stream) {
    const auto blocks_of = [&](int64_t units) { return (units * a.columns + SUM_WARPS - 1) / SUM_WARPS; };
    const int64_t pieces = blocks_of(a.pieces), runs = blocks_of((static_cast<int64_t>(a.n) + TILE - 1) / TILE);
    const int64_t all = (pieces + runs + zero_blocks) * M;
    if (all == 0) return cudaSuccess;
    if (all > 0x7fffffff) return cudaErrorInvalidConfiguration;   // (beyond any memory)
    const SumBlocks blocks{static_cast<unsigned>(pieces), static_cast<unsigned>(runs), static_cast<unsigned>(zero_blocks), rows};
    return launch_op(grad_sums_kernel<ST, GT, N>, dim3(static_cast<unsigned>(all)), dim3(SUM_THREADS), 0, true, stream, a, blocks, M);
}

template <typename GT>
cudaError_t launch_sort(const EmbedGradArgs &a, int M, int64_t zero_blocks, int rows, cudaStream_t stream) {
    const size_t smem = static_cast<size_t>(SORT_WARPS + 2) * a.keys * sizeof(int);
    const int64_t all = ((int64_t{1} << a.bits) + zero_blocks) * M;
    if (all > 0x7fffffff) return cudaErrorInvalidConfiguration;
    const auto kernel = a.n <= SORT_CACHED ? (a.tokens.wide ? token_sort_kernel<true, true, GT> : token_sort_kernel<true, false, GT>)
                                           : (a.tokens.wide ? token_sort_kernel<false, true, GT> : token_sort_kernel<false, false, GT>);
    return launch_op(kernel, dim3(static_cast<unsigned>(all)), dim3(SORT_THREADS), smem, true, stream, a, M, static_cast<unsigned>(zero_blocks), rows);
}

// Columns at a time: eight where every row of both sides begins on a 16-byte boundary, two where it begins on one of two elements, else one.
int columns_at_a_time(const EmbedGradArgs &a, int M, bool dout_bf16, bool grad_bf16) {
    const long long ssz = dout_bf16 ? 2 : 4, gsz = grad_bf16 ? 2 : 4;
    const uintptr_t from = reinterpret_cast<uintptr_t>(a.dout) | static_cast<uintptr_t>(a.ds0 * ssz) | static_cast<uintptr_t>(a.ds1 * ssz);
    uintptr_t to = static_cast<uintptr_t>(a.width * gsz);
    for (int m = 0; m < M; ++m) to |= reinterpret_cast<uintptr_t>(a.g[m]);
    if (((from | to) & 15u) == 0 && a.width % 8 == 0) return 8;
    return (from & (2 * ssz - 1)) == 0 && (to & (2 * gsz - 1)) == 0 && a.width % 2 == 0 ? 2 : 1;
}

template <typename ST, typename GT>
cudaError_t launch_sums(const EmbedGradArgs &a, int M, int columns, int64_t zero_blocks, int rows, cudaStream_t stream) {
    return (columns == 8 ? launch_sums<ST, GT, 8> : columns == 2 ? launch_sums<ST, GT, 2> : launch_sums<ST, GT, 1>)(a, M, zero_blocks, rows, stream);
}

}  // namespace

cudaError_t launch_embed(const EmbedArgs &a, int M, bool bf16, cudaStream_t stream) {
    // a warp per row, or the whole block where there are few
    const unsigned lanes = static_cast<int64_t>(a.n) * M >= 4 * 148 * 4 ? 32 : EMBED_THREADS;
    const dim3 threads(lanes, EMBED_THREADS / lanes), grid((a.n + threads.y - 1) / threads.y, M);
    return launch_op(bf16 ? embed_kernel<__nv_bfloat16> : embed_kernel<float>, grid, threads, 0, true, stream, a);
}

int64_t plan_embed_grad(EmbedGradArgs &a, int M, char *work) {
    // As few blocks as their counters allow (each goes over all tokens), but enough of them.
    a.bits = 0;
    const auto keys = [&] { return ((a.vocab - 1) >> a.bits) + 1; };
    while (keys() > SORT_KEYS || (keys() > 64 && (static_cast<int64_t>(M) << a.bits) < 128)) ++a.bits;
    a.keys = keys();
    a.piece = 32;
    while (16LL * a.piece * a.piece < a.n) a.piece *= 2;
    a.pieces = a.n < a.piece ? 0 : (a.n - 1) / a.piece + 1;   // (a number is below n / piece: its place lies in a run)
    a.row = (static_cast<int64_t>(a.width) + 7) & ~int64_t{7};
    a.columns = static_cast<int>((static_cast<int64_t>(a.width) + 31) / 32);   // (as many as there can be: of one column a lane)
    int64_t at = 0;
    const auto take = [&](int64_t bytes) {
        char *p = work ? work + at : nullptr;
        at += (bytes + 255) & ~int64_t{255};
        return p;
    };
    a.seen = reinterpret_cast<unsigned char *>(take(static_cast<int64_t>(M) * a.vocab));
    a.places = reinterpret_cast<int4 *>(take(static_cast<int64_t>(M) * a.n * 16));
    a.count = reinterpret_cast<int *>(take(static_cast<int64_t>(M) * 4));
    a.tickets = reinterpret_cast<int *>(take(static_cast<int64_t>(M) * a.pieces * a.columns * 4));
    a.partial = reinterpret_cast<float *>(take(static_cast<int64_t>(M) * a.pieces * a.row * 4));
    return at;
}

cudaError_t launch_embed_grad(EmbedGradArgs a, int M, bool dout_bf16, bool grad_bf16, cudaStream_t stream, int *launches) {
    const int columns = columns_at_a_time(a, M, dout_bf16, grad_bf16);
    a.columns = (a.width + 32 * columns - 1) / (32 * columns);
    // Zeros: written while the tokens are sorted, by blocks that look all of them up themselves; beyond ZEROS_AHEAD tokens, where that takes
    // too long, behind the sort, which knows.  Rows per block: as many as have 300 KB of zeros to
    // write (the more, the fewer blocks go over the tokens, and the later DRAM has something to do), fewer where that leaves too few blocks.
    int rows = MOST_ZERO_ROWS;
    while (rows > ZERO_ROWS && static_cast<int64_t>(rows) * a.width * (grad_bf16 ? 2 : 4) > ZERO_BYTES) rows /= 2;
    while (rows > SORT_WARPS && static_cast<int64_t>(a.vocab) * M < static_cast<int64_t>(rows) * 148 * 4) rows /= 2;
    if (a.n > ZEROS_AHEAD && rows > 32 * SUM_WARPS) rows = 32 * SUM_WARPS;
    const int64_t zero_blocks = a.accumulate ? 0 : (static_cast<int64_t>(a.vocab) + rows - 1) / rows;
    const int64_t ahead = a.n <= ZEROS_AHEAD ? zero_blocks : 0, behind = zero_blocks - ahead;
    cudaError_t e = grad_bf16 ? launch_sort<__nv_bfloat16>(a, M, ahead, rows, stream) : launch_sort<float>(a, M, ahead, rows, stream);
    if (e != cudaSuccess) return e;
    *launches = 1;
    using bf = __nv_bfloat16;
    if (dout_bf16) e = (grad_bf16 ? launch_sums<bf, bf> : launch_sums<bf, float>)(a, M, columns, behind, rows, stream);
    else e = (grad_bf16 ? launch_sums<float, bf> : launch_sums<float, float>)(a, M, columns, behind, rows, stream);
    if (e == cudaSuccess) *launches = 2;
    return e;
}

}  // namespace desloc
