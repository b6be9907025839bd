// Embedding lookup from the workers' replicas, and its gradient by sorted tokens.
#include "desloc_ops.cuh"

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
// its own and those of the blocks in front of it, and writes its part of the order.  No block waits for another.
constexpr int SORT_THREADS = 512, SORT_WARPS = SORT_THREADS / 32, SORT_AHEAD = 4;
constexpr int SORT_KEYS = 760;   // most numbers that a block tells apart: counters of 47.5 KB

__global__ void __launch_bounds__(SORT_THREADS) token_sort_kernel(const EmbedGradArgs a) {
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
    const long long share = (static_cast<long long>(a.n) + SORT_THREADS - 1) / SORT_THREADS * 32;
    const long long lo = min(static_cast<long long>(a.n), warp * share), hi = min(static_cast<long long>(a.n), lo + share);
    const long long t0 = m * a.tokens.s0;
    int before = 0;
    for (long long i0 = lo; i0 < hi; i0 += 32 * SORT_AHEAD) {
        int t[SORT_AHEAD];
#pragma unroll
        for (int k = 0; k < SORT_AHEAD; ++k) {
            const long long i = i0 + 32 * k + lane;
            t[k] = i < hi ? token_at(a.tokens, t0 + i * a.tokens.s1, a.vocab) : -1;
        }
#pragma unroll
        for (int k = 0; k < SORT_AHEAD; ++k) {
            if (t[k] < 0) continue;
            if ((t[k] & mask) == b) atomicAdd(&mine[t[k] >> a.bits], 1);
            before += (t[k] & mask) < b;
        }
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) before += __shfl_down_sync(0xffffffffu, before, off);
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
    for (long long i0 = lo; i0 < hi; i0 += 32 * SORT_AHEAD) {
        int t[SORT_AHEAD];
#pragma unroll
        for (int k = 0; k < SORT_AHEAD; ++k) {
            const long long i = i0 + 32 * k + lane;
            t[k] = i < hi ? token_at(a.tokens, t0 + i * a.tokens.s1, a.vocab) : -1;
        }
#pragma unroll
        for (int k = 0; k < SORT_AHEAD; ++k) {
            const bool is = t[k] >= 0 && (t[k] & mask) == b;
            const unsigned who = __ballot_sync(0xffffffffu, is);
            if (is) {
                const int key = t[k] >> a.bits;
                const unsigned same = __match_any_sync(who, key);
                const int rank = __popc(same & ((1u << lane) - 1));
                const int at = mine[key];
                order[at + rank] = static_cast<int>(i0 + 32 * k + lane);
                __syncwarp(who);
                if (rank == 0) mine[key] = at + __popc(same);
            }
            __syncwarp();
        }
    }
}

// ---- sums --------------------------------------------------------------------------------------------
// A run (the positions of one token) of `piece` or more tokens is cut into floor(length / piece) pieces of nearly equal length, summed by
// a block each; the row's sum adds them in order.  Piece j of a run that begins at place s has number ceil(s / piece) + j: no two
// runs' numbers meet, because ceil(a + b) >= ceil(a) + floor(b), and place number * piece lies in the run.
struct Pieces {
    int first, n;
    __device__ __forceinline__ Pieces(const EmbedGradArgs &a, int2 run)
        : first(static_cast<int>((static_cast<long long>(run.x) + a.piece - 1) / a.piece)), n(run.y / a.piece) {}
};

template <int N>
__device__ __forceinline__ void add_to(float (&acc)[N], const float (&f)[N]) {
#pragma unroll
    for (int e = 0; e < N; ++e) acc[e] += f[e];
}

constexpr int PIECE_WARPS = 8;

template <typename ST, int N>
__global__ void __launch_bounds__(32 * PIECE_WARPS) run_pieces_kernel(const EmbedGradArgs a) {
    __shared__ float sums[PIECE_WARPS][32 * N];
    begin_and_let_next_begin();
    wait_for_earlier_kernels();
    const int p = blockIdx.x, m = blockIdx.z, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long place = static_cast<long long>(p) * a.piece;
    if (place >= a.count[m]) return;
    const int *order = a.order + static_cast<long long>(m) * a.n;
    const int tok = token_at(a.tokens, m * a.tokens.s0 + order[place] * a.tokens.s1, a.vocab);
    const int2 run = a.range[static_cast<long long>(m) * a.vocab + tok];
    const Pieces pc(a, run);
    const int j = p - pc.first;
    if (j < 0 || j >= pc.n) return;
    const int lo = run.x + static_cast<int>(static_cast<long long>(run.y) * j / pc.n);
    const int hi = run.x + static_cast<int>(static_cast<long long>(run.y) * (j + 1) / pc.n);
    const int col = static_cast<int>((blockIdx.y * 32 + lane) * N);
    float acc[N] = {};
    if (col < a.width) {
        const ST *base = static_cast<const ST *>(a.dout) + m * a.ds0 + col;
        for (int i0 = lo + warp; i0 < hi; i0 += 4 * PIECE_WARPS) {
            float f[4][N];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (i0 + k * PIECE_WARPS < hi) load_values(base + order[i0 + k * PIECE_WARPS] * a.ds1, f[k]);
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (i0 + k * PIECE_WARPS < hi) add_to(acc, f[k]);
        }
    }
#pragma unroll
    for (int e = 0; e < N; ++e) sums[warp][e * 32 + lane] = acc[e];
    __syncthreads();
    float *out = a.partial + (static_cast<long long>(m) * a.pieces + p) * a.row + static_cast<long long>(blockIdx.y) * 32 * N;
    for (int c = threadIdx.x; c < 32 * N; c += 32 * PIECE_WARPS) {   // column c = lane * N + element
        if (blockIdx.y * 32 * N + c >= static_cast<unsigned>(a.width)) break;
        const int at = (c % N) * 32 + c / N;
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < PIECE_WARPS; ++w) t += sums[w][at];
        out[c] = t;
    }
}

// The rows of the gradient.  A warp takes 32 * N columns of a row: the run's rows of dout in order, or the sums of its pieces, or
// nothing but zeros to write.  Bound: HBM writes of the whole gradient.
constexpr int ROWS_THREADS = 256, ROWS_PER_BLOCK = 16;

template <typename ST, typename GT, int N>
__global__ void __launch_bounds__(ROWS_THREADS) grad_rows_kernel(const EmbedGradArgs a) {
    __shared__ int2 runs[ROWS_PER_BLOCK];
    begin_and_let_next_begin();
    const int m = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int v0 = static_cast<int>(blockIdx.x) * ROWS_PER_BLOCK, rows = min(ROWS_PER_BLOCK, a.vocab - v0);
    wait_for_earlier_kernels();
    if (static_cast<int>(threadIdx.x) < rows) runs[threadIdx.x] = a.range[static_cast<long long>(m) * a.vocab + v0 + threadIdx.x];
    __syncthreads();
    const int *order = a.order + static_cast<long long>(m) * a.n;
    const int parts = (a.width + 32 * N - 1) / (32 * N);
    for (long long u = warp; u < static_cast<long long>(rows) * parts; u += ROWS_THREADS / 32) {
        const int r = static_cast<int>(u / parts), col = static_cast<int>((u - static_cast<long long>(r) * parts) * 32 + lane) * N;
        const int2 run = runs[r];
        if (col >= a.width || (run.y == 0 && a.accumulate)) continue;
        float acc[N] = {};
        if (run.y >= a.piece) {
            const Pieces pc(a, run);
            const float *sum = a.partial + (static_cast<long long>(m) * a.pieces + pc.first) * a.row + col;
            for (int j0 = 0; j0 < pc.n; j0 += 4) {
                float f[4][N];
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (j0 + k < pc.n) load_values(sum + (j0 + k) * a.row, f[k]);
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (j0 + k < pc.n) add_to(acc, f[k]);
            }
        } else {
            const ST *base = static_cast<const ST *>(a.dout) + m * a.ds0 + col;
            for (int i0 = run.x; i0 < run.x + run.y; i0 += 4) {
                float f[4][N];
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (i0 + k < run.x + run.y) load_values(base + order[i0 + k] * a.ds1, f[k]);
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (i0 + k < run.x + run.y) add_to(acc, f[k]);
            }
        }
        GT *out = static_cast<GT *>(a.g[m]) + static_cast<long long>(v0 + r) * a.width + col;
        float old[N] = {};
        if (a.accumulate) load_values(out, old);
#pragma unroll
        for (int e = 0; e < N; ++e) acc[e] = a.accumulate ? fmaf(acc[e], a.scale, old[e]) : acc[e] * a.scale;
        store_values(out, acc);
    }
}

template <typename ST, typename GT, int N>
cudaError_t launch_sums(const EmbedGradArgs &a, int M, cudaStream_t stream, int *launches) {
    const unsigned cols = static_cast<unsigned>((a.width + 32 * N - 1) / (32 * N));
    if (a.pieces > 0) {
        const cudaError_t e = launch_op(run_pieces_kernel<ST, N>, dim3(a.pieces, cols, M), dim3(32 * PIECE_WARPS), 0, true, stream, a);
        if (e != cudaSuccess) return e;
        *launches += 1;
    }
    const cudaError_t e = launch_op(grad_rows_kernel<ST, GT, N>, dim3((a.vocab + ROWS_PER_BLOCK - 1) / ROWS_PER_BLOCK, M), dim3(ROWS_THREADS), 0, true, stream, a);
    if (e == cudaSuccess) *launches += 1;
    return e;
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
    a.piece = 64;
    while (4LL * a.piece * a.piece < a.n) a.piece *= 2;
    a.pieces = a.n < a.piece ? 0 : (a.n - 1) / a.piece + 1;   // (a number is below n / piece: its place lies in a run)
    a.row = (static_cast<int64_t>(a.width) + 7) & ~int64_t{7};
    int64_t at = 0;
    const auto take = [&](int64_t bytes) {
        char *p = work ? work + at : nullptr;
        at += (bytes + 255) & ~int64_t{255};
        return p;
    };
    a.range = reinterpret_cast<int2 *>(take(static_cast<int64_t>(M) * a.vocab * 8));
    a.order = reinterpret_cast<int *>(take(static_cast<int64_t>(M) * a.n * 4));
    a.count = reinterpret_cast<int *>(take(static_cast<int64_t>(M) * 4));
    a.partial = reinterpret_cast<float *>(take(static_cast<int64_t>(M) * a.pieces * a.row * 4));
    return at;
}

cudaError_t launch_embed_grad(const EmbedGradArgs &a, int M, bool dout_bf16, bool grad_bf16, cudaStream_t stream, int *launches) {
    const size_t smem = static_cast<size_t>(SORT_WARPS) * a.keys * sizeof(int);
    const cudaError_t e = launch_op(token_sort_kernel, dim3(1u << a.bits, M), dim3(SORT_THREADS), smem, true, stream, a);
    if (e != cudaSuccess) return e;
    *launches = 1;
    // eight columns at a time where every row of both sides begins on a 16-byte boundary
    const long long ssz = dout_bf16 ? 2 : 4, gsz = grad_bf16 ? 2 : 4;
    uintptr_t off = reinterpret_cast<uintptr_t>(a.dout) | static_cast<uintptr_t>(a.ds0 * ssz) | static_cast<uintptr_t>(a.ds1 * ssz) |
                    static_cast<uintptr_t>(a.width * gsz);
    for (int m = 0; m < M; ++m) off |= reinterpret_cast<uintptr_t>(a.g[m]);
    const bool wide = (off & 15u) == 0 && a.width % 8 == 0;
    using bf = __nv_bfloat16;
    if (dout_bf16)
        return grad_bf16 ? (wide ? launch_sums<bf, bf, 8> : launch_sums<bf, bf, 1>)(a, M, stream, launches)
                         : (wide ? launch_sums<bf, float, 8> : launch_sums<bf, float, 1>)(a, M, stream, launches);
    return grad_bf16 ? (wide ? launch_sums<float, bf, 8> : launch_sums<float, bf, 1>)(a, M, stream, launches)
                     : (wide ? launch_sums<float, float, 8> : launch_sums<float, float, 1>)(a, M, stream, launches);
}

}  // namespace desloc
