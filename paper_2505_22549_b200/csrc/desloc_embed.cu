// Embedding lookup from the workers' replicas, and its gradient by sorted tokens.
#include "desloc_ops.cuh"

#include <type_traits>

namespace desloc {

namespace {

// ---- lookup ------------------------------------------------------------------------------------------
// out[m, i, :] = scale * x^m[token(m, i), :].  Bound: HBM, 4 bytes read (rows that occur again come from L2) and 2 or 4 written per
// element.  `blockDim.x` lanes take a row, four 16-byte loads in flight each.
constexpr int EMBED_THREADS = 128;

template <typename OT>
__global__ void __launch_bounds__(EMBED_THREADS) embed_kernel(const EmbedArgs a) {
    begin_and_let_next_begin();
    const int m = blockIdx.y, lanes = blockDim.x;
    const int i = static_cast<int>(blockIdx.x * blockDim.y + threadIdx.y);
    wait_for_earlier_kernels();
    if (i >= a.n) return;
    const int tok = token_at(a.tokens, m * a.tokens.s0 + i * a.tokens.s1, a.vocab);
    OT *out = static_cast<OT *>(a.out) + m * a.os0 + i * a.os1;
    const float *row = a.x[static_cast<long long>(m) * a.x_stride] + static_cast<long long>(max(tok, 0)) * a.width;
    const bool none = tok < 0;
    if (a.width % 4 == 0 && (reinterpret_cast<uintptr_t>(row) & 15u) == 0 && (reinterpret_cast<uintptr_t>(out) & (4 * sizeof(OT) - 1)) == 0) {
        for (int c = threadIdx.x; c < a.width / 4; c += 4 * lanes) {
            float f[4][4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (!none && c + k * lanes < a.width / 4) load_values(row + 4 * (c + k * lanes), f[k]);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (c + k * lanes >= a.width / 4) break;
#pragma unroll
                for (int e = 0; e < 4; ++e) f[k][e] = none ? 0.f : f[k][e] * a.scale;
                store_values(out + 4 * (c + k * lanes), f[k]);
            }
        }
    } else {
        for (int c = threadIdx.x; c < a.width; c += lanes) {
            const float f[1] = {none ? 0.f : row[c] * a.scale};
            store_values(out + c, f);
        }
    }
}

// ---- sort --------------------------------------------------------------------------------------------
// Stable counting sort of a worker's tokens, a block for each value of the tokens' last bits: it goes over all of them twice, counts
// its own and those of the blocks in front of it, and writes its part of the order and its runs (a run: the places of one token).  No
// block waits for another.  Bound: latency; up to SORT_CACHED tokens stay in registers between the two times.
constexpr int SORT_THREADS = 512, SORT_WARPS = SORT_THREADS / 32, SORT_AHEAD = 16;
constexpr int SORT_CACHED = SORT_THREADS * SORT_AHEAD;
constexpr int SORT_KEYS = 760;   // most numbers that a block tells apart: counters of 47.5 KB

// A run of `piece` or more places is cut into floor(length / piece) pieces of nearly equal length, summed by a block each.  Piece j of
// a run that begins at place s has number ceil(s / piece) + j: no two runs' numbers meet, because ceil(a + b) >= ceil(a) + floor(b), and
// place number * piece lies in the run.
struct Pieces {
    int first, n;
    __device__ __forceinline__ Pieces(const EmbedGradArgs &a, int start, int length)
        : first((start + a.piece - 1) / a.piece), n(length / a.piece) {}
};

// WIDE: 64-bit token numbers.
template <bool CACHED, bool WIDE>
__global__ void __launch_bounds__(SORT_THREADS) token_sort_kernel(const __grid_constant__ EmbedGradArgs a) {
    using Number = std::conditional_t<WIDE, long long, int>;
    extern __shared__ int hist[];   // [warp][key]: counts, then places
    __shared__ int s_warp[SORT_WARPS];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int b = blockIdx.x, m = blockIdx.y, mask = (1 << a.bits) - 1;
    int *mine = hist + warp * a.keys;
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
        Number v[SORT_AHEAD];
        const Number *p = tokens + (i0 + lane) * a.tokens.s1;
        const long long step = 32 * a.tokens.s1;
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
            a.range[static_cast<long long>(m) * a.vocab + v] = make_int2(at, total);
            if (total >= a.piece) {
                const long long ticket = static_cast<long long>(m) * a.pieces + Pieces(a, at, total).first;
                for (int c = 0; c < a.columns; ++c) a.tickets[ticket * a.columns + c] = 0;
            }
            if (total > 0)
#pragma unroll
                for (int w = 0; w < SORT_WARPS; ++w) {
                    const int c = hist[w * a.keys + key];
                    hist[w * a.keys + key] = at;
                    at += c;
                }
        }
        base += all;
    }
    if (b == mask && tid == 0) a.count[m] = base;
    __syncthreads();
    int *order = a.order + static_cast<long long>(m) * a.n;
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
                order[at + rank] = i0 + 32 * k + lane;
                __syncwarp(who);
                if (rank == 0) mine[key] = at + __popc(same);
            }
            __syncwarp();
        }
    }
}

// ---- sums --------------------------------------------------------------------------------------------
// One launch, blocks of two kinds: pieces of long runs, and rows of the gradient in order: the sums of short runs, and the zeros of rows without a
// token, which are most of a large vocabulary.  Bound: HBM, rows of dout read and the gradient written.
constexpr int SUM_THREADS = 256, SUM_WARPS = SUM_THREADS / 32;
constexpr int MOST_ROWS = 64;      // rows of the gradient that a block takes, at most
constexpr int PIECES_ASKED = 4;    // piece numbers that a block looks up: most stand for none

// acc += rows order[lo], order[lo + step], ... below hi, N columns from `base` on, in order.
template <int N, typename ST>
__device__ __forceinline__ void add_rows(float (&acc)[N], const ST *base, long long stride, const int *order, int lo, int hi, int step) {
    constexpr int AHEAD = N * sizeof(ST) > 16 ? 2 : 4;
    using Piece = std::conditional_t<N == 1, ST, uint4>;
    constexpr int WORDS = N == 1 ? 1 : N * static_cast<int>(sizeof(ST)) / 16;   // (unpacked when they are added: a row in flight costs four registers)
    for (int i0 = lo; i0 < hi; i0 += AHEAD * step) {
        Piece w[AHEAD][WORDS];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (i0 + k * step < hi) {
                const Piece *row = reinterpret_cast<const Piece *>(base + order[i0 + k * step] * stride);
#pragma unroll
                for (int q = 0; q < WORDS; ++q) w[k][q] = row[q];
            }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (i0 + k * step < hi) {
                float f[N];
                load_values(reinterpret_cast<const ST *>(w[k]), f);
#pragma unroll
                for (int e = 0; e < N; ++e) acc[e] += f[e];
            }
    }
}

template <int N, typename GT>
__device__ __forceinline__ void write_sum(const EmbedGradArgs &a, GT *out, float (&acc)[N]) {
    float old[N] = {};
    if (a.accumulate) load_values(out, old);
#pragma unroll
    for (int e = 0; e < N; ++e) acc[e] = a.accumulate ? fmaf(acc[e], a.scale, old[e]) : acc[e] * a.scale;
    store_values(out, acc);
}

// Sums of the warps' accs, in their order, N columns per lane: column lane * N + e of the block is sums[...][e * 32 + lane].  In warp 0.
template <int N>
__device__ __forceinline__ void join_warps(float (&acc)[N], float (*sums)[32 * N]) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int e = 0; e < N; ++e) sums[warp][e * 32 + lane] = acc[e];
    __syncthreads();
    if (warp == 0)
#pragma unroll
        for (int e = 0; e < N; ++e) {
            acc[e] = 0.f;
#pragma unroll
            for (int w = 0; w < SUM_WARPS; ++w) acc[e] += sums[w][e * 32 + lane];
        }
}

// A piece of a long run: place in the run's order, token, first place and length of the run.
struct Piece {
    int j, tok, start, length;
};

// Piece number p of worker m; j < 0 where it stands for none.
__device__ __forceinline__ Piece find_piece(const EmbedGradArgs &a, int m, int p) {
    const long long place = static_cast<long long>(p) * a.piece;
    if (p >= a.pieces || place >= a.count[m]) return {-1, 0, 0, 0};
    const int position = a.order[static_cast<long long>(m) * a.n + place];
    const int tok = token_at(a.tokens, m * a.tokens.s0 + position * a.tokens.s1, a.vocab);
    const int2 run = a.range[static_cast<long long>(m) * a.vocab + tok];
    const Pieces pc(a, run.x, run.y);
    const int j = p - pc.first;
    return {j < pc.n ? j : -1, tok, run.x, run.y};
}

// 32 * N columns of a piece.  The last block of a run's to arrive adds the pieces in their order and writes the row.
template <typename ST, typename GT, int N>
__device__ __forceinline__ void sum_piece(const EmbedGradArgs &a, int m, const Piece &q, int c, float (*sums)[32 * N]) {
    __shared__ int s_last;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const Pieces pc(a, q.start, q.length);
    const int lo = q.start + static_cast<int>(static_cast<long long>(q.length) * q.j / pc.n);
    const int hi = q.start + static_cast<int>(static_cast<long long>(q.length) * (q.j + 1) / pc.n);
    const int col = (c * 32 + lane) * N;
    const bool in = col < a.width;
    float acc[N] = {};
    if (in) add_rows(acc, static_cast<const ST *>(a.dout) + m * a.ds0 + col, a.ds1, a.order + static_cast<long long>(m) * a.n, lo + warp, hi, SUM_WARPS);
    join_warps<N>(acc, sums);
    GT *out = static_cast<GT *>(a.g[m]) + static_cast<long long>(q.tok) * a.width + col;
    if (pc.n > 1) {
        float *const part = a.partial + (static_cast<long long>(m) * a.pieces + pc.first) * a.row + col;
        if (warp == 0) {
            if (in) store_values(part + q.j * a.row, acc);
            __threadfence();
            __syncwarp();
            if (lane == 0) s_last = atomicAdd(&a.tickets[(static_cast<long long>(m) * a.pieces + pc.first) * a.columns + c], 1) == pc.n - 1;
        }
        __syncthreads();
        if (!s_last) return;
        __threadfence();
#pragma unroll
        for (int e = 0; e < N; ++e) acc[e] = 0.f;
        if (in)
            for (int k0 = warp; k0 < pc.n; k0 += 2 * SUM_WARPS) {
                float f[2][N];
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    if (k0 + k * SUM_WARPS < pc.n)
#pragma unroll
                        for (int e = 0; e < N; ++e) f[k][e] = __ldcg(part + (k0 + k * SUM_WARPS) * a.row + e);
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    if (k0 + k * SUM_WARPS < pc.n)
#pragma unroll
                        for (int e = 0; e < N; ++e) acc[e] += f[k][e];
            }
        join_warps<N>(acc, sums);
    }
    if (warp == 0 && in) write_sum<N>(a, out, acc);
}

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

template <typename ST, typename GT, int N>
__global__ void __launch_bounds__(SUM_THREADS, 5) grad_sums_kernel(const __grid_constant__ EmbedGradArgs a, unsigned piece_blocks, int block_rows) {
    __shared__ float sums[SUM_WARPS][32 * N];
    __shared__ Piece s_piece[PIECES_ASKED];
    __shared__ int4 s_run[MOST_ROWS];   // row of the block, first place, length
    __shared__ int s_runs;
    __shared__ unsigned s_none[MOST_ROWS / 32];
    begin_and_let_next_begin();
    const int m = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) s_runs = 0;
    wait_for_earlier_kernels();
    if (blockIdx.x < piece_blocks) {
        const int c = static_cast<int>(blockIdx.x % a.columns), p0 = static_cast<int>(blockIdx.x / a.columns) * PIECES_ASKED;
        if (tid < PIECES_ASKED) s_piece[tid] = find_piece(a, m, p0 + tid);
        __syncthreads();
        for (int k = 0; k < PIECES_ASKED; ++k) {
            const Piece q = s_piece[k];
            if (q.j < 0) continue;
            sum_piece<ST, GT, N>(a, m, q, c, sums);
            __syncthreads();   // (what it shares is free again)
        }
        return;
    }
    const int v0 = static_cast<int>(blockIdx.x - piece_blocks) * block_rows, rows = min(block_rows, a.vocab - v0);
    __syncthreads();
    if (tid < MOST_ROWS) {
        int2 run = make_int2(0, -1);
        if (tid < rows) run = a.range[static_cast<long long>(m) * a.vocab + v0 + tid];
        const unsigned none = __ballot_sync(0xffffffffu, run.y == 0);
        if (lane == 0) s_none[warp] = none;
        if (run.y > 0 && run.y < a.piece) s_run[atomicAdd(&s_runs, 1)] = make_int4(tid, run.x, run.y, 0);
    }
    __syncthreads();
    GT *const out = static_cast<GT *>(a.g[m]) + static_cast<long long>(v0) * a.width;
    if (!a.accumulate) {
        // neighbouring rows of a warp's at once
        const int each = (block_rows + SUM_WARPS - 1) / SUM_WARPS, r0 = warp * each;   // (each: 1, 2, 4 or 8)
        unsigned todo = r0 < MOST_ROWS ? s_none[r0 / 32] >> (r0 % 32) & ((1u << each) - 1) : 0;
        while (todo) {
            const int r = __ffs(todo) - 1, n = __ffs(~(todo >> r)) - 1;
            zero_span(reinterpret_cast<char *>(out + static_cast<long long>(r0 + r) * a.width), n * (static_cast<long long>(a.width) * sizeof(GT)));
            todo &= ~(((1u << n) - 1) << r);
        }
    }
    const unsigned across = static_cast<unsigned>((a.width + N - 1) / N), units = static_cast<unsigned>(s_runs) * across;
    for (unsigned f = tid; f < units; f += SUM_THREADS) {
        const unsigned i = f / across;
        const int col = static_cast<int>(f - i * across) * N;
        const int4 run = s_run[i];
        float acc[N] = {};
        add_rows(acc, static_cast<const ST *>(a.dout) + m * a.ds0 + col, a.ds1, a.order + static_cast<long long>(m) * a.n, run.y, run.y + run.z, 1);
        write_sum<N>(a, out + static_cast<long long>(run.x) * a.width + col, acc);
    }
}

template <typename ST, typename GT, int N>
cudaError_t launch_sums(const EmbedGradArgs &a, int M, cudaStream_t stream) {
    // rows per block: as many as leave several rounds of blocks
    int rows = MOST_ROWS;
    while (rows > 1 && static_cast<int64_t>(a.vocab) * M < static_cast<int64_t>(rows) * 148 * 16) rows /= 2;
    const int64_t piece_blocks = (static_cast<int64_t>(a.pieces) + PIECES_ASKED - 1) / PIECES_ASKED * a.columns;
    const int64_t blocks = piece_blocks + (static_cast<int64_t>(a.vocab) + rows - 1) / rows;
    if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;   // (beyond any memory)
    return launch_op(grad_sums_kernel<ST, GT, N>, dim3(static_cast<unsigned>(blocks), M), dim3(SUM_THREADS), 0, true, stream, a,
                     static_cast<unsigned>(piece_blocks), rows);
}

// Eight columns at a time where every row of both sides begins on a 16-byte boundary.
bool eight_columns(const EmbedGradArgs &a, int M, bool dout_bf16, bool grad_bf16) {
    const long long ssz = dout_bf16 ? 2 : 4, gsz = grad_bf16 ? 2 : 4;
    uintptr_t off = reinterpret_cast<uintptr_t>(a.dout) | static_cast<uintptr_t>(a.ds0 * ssz) | static_cast<uintptr_t>(a.ds1 * ssz) |
                    static_cast<uintptr_t>(a.width * gsz);
    for (int m = 0; m < M; ++m) off |= reinterpret_cast<uintptr_t>(a.g[m]);
    return (off & 15u) == 0 && a.width % 8 == 0;
}

}  // namespace

cudaError_t launch_embed(const EmbedArgs &a, int M, bool bf16, cudaStream_t stream) {
    // a warp per row, or the whole block where there are few
    const unsigned lanes = static_cast<int64_t>(a.n) * M >= 4 * 148 * 4 ? 32 : EMBED_THREADS;
    const dim3 threads(lanes, EMBED_THREADS / lanes), grid((a.n + threads.y - 1) / threads.y, M);
    return launch_op(bf16 ? embed_kernel<__nv_bfloat16> : embed_kernel<float>, grid, threads, 0, true, stream, a);
}

int64_t plan_embed_grad(EmbedGradArgs &a, int M, char *work) {
    a.bits = 0;
    while (((a.vocab - 1) >> a.bits) + 1 > SORT_KEYS) ++a.bits;
    a.keys = ((a.vocab - 1) >> a.bits) + 1;
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
    a.range = reinterpret_cast<int2 *>(take(static_cast<int64_t>(M) * a.vocab * 8));
    a.order = reinterpret_cast<int *>(take(static_cast<int64_t>(M) * a.n * 4));
    a.count = reinterpret_cast<int *>(take(static_cast<int64_t>(M) * 4));
    a.tickets = reinterpret_cast<int *>(take(static_cast<int64_t>(M) * a.pieces * a.columns * 4));
    a.partial = reinterpret_cast<float *>(take(static_cast<int64_t>(M) * a.pieces * a.row * 4));
    return at;
}

cudaError_t launch_embed_grad(EmbedGradArgs a, int M, bool dout_bf16, bool grad_bf16, cudaStream_t stream, int *launches) {
    const bool wide = eight_columns(a, M, dout_bf16, grad_bf16);
    a.columns = (a.width + (wide ? 255 : 31)) / (wide ? 256 : 32);
    const size_t smem = static_cast<size_t>(SORT_WARPS) * a.keys * sizeof(int);
    const auto sort = a.n <= SORT_CACHED ? (a.tokens.wide ? token_sort_kernel<true, true> : token_sort_kernel<true, false>)
                                         : (a.tokens.wide ? token_sort_kernel<false, true> : token_sort_kernel<false, false>);
    cudaError_t e = launch_op(sort, dim3(1u << a.bits, M), dim3(SORT_THREADS), smem, true, stream, a);
    if (e != cudaSuccess) return e;
    *launches = 1;
    using bf = __nv_bfloat16;
    if (dout_bf16)
        e = grad_bf16 ? (wide ? launch_sums<bf, bf, 8> : launch_sums<bf, bf, 1>)(a, M, stream)
                      : (wide ? launch_sums<bf, float, 8> : launch_sums<bf, float, 1>)(a, M, stream);
    else
        e = grad_bf16 ? (wide ? launch_sums<float, bf, 8> : launch_sums<float, bf, 1>)(a, M, stream)
                      : (wide ? launch_sums<float, float, 8> : launch_sums<float, float, 1>)(a, M, stream);
    if (e == cudaSuccess) *launches = 2;
    return e;
}

}  // namespace desloc
