// Log probabilities of given tokens with entropy and the largest alternatives, and their gradient.
#include "desloc_ops.cuh"

#include <cfloat>

#include "desloc_internal.cuh"

namespace desloc {

namespace {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float FAR_BELOW = -1e30f;   // an exponent of 2 that stands for minus infinity where 0 * infinity may not arise

// 2^t, relative error 2^-22; 0 below -126.
__device__ __forceinline__ float exp2_fast(float t) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(t));
    return r;
}

// Running softmax of a part of a row: largest value m, S = sum of 2^t and A = sum of t 2^t with t = (x - m) log2 e.
// Parts without values (or of nothing but -inf) have m = -FLT_MAX and S = 0; NaN and +inf end in a NaN S.
struct Running {
    float m, S, A;
};

template <bool ENT>
__device__ __forceinline__ void raise_to(Running &r, float m) {
    const float d = fmaxf((r.m - m) * LOG2E, FAR_BELOW), f = exp2_fast(d);
    if constexpr (ENT) r.A = f * fmaf(r.S, d, r.A);
    r.S *= f;
    r.m = m;
}

template <bool ENT>
__device__ __forceinline__ Running join(Running a, Running b) {
    const float m = fmaxf(a.m, b.m);
    raise_to<ENT>(a, m);
    raise_to<ENT>(b, m);
    return {m, a.S + b.S, ENT ? a.A + b.A : 0.f};
}

template <bool ENT, int N>
__device__ __forceinline__ void take(Running &r, const float (&f)[N]) {
    float top = f[0];
#pragma unroll
    for (int k = 1; k < N; ++k) top = fmaxf(top, f[k]);
    if (top > r.m) raise_to<ENT>(r, top);
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const float t = (f[k] - r.m) * LOG2E, e = exp2_fast(t);
        r.S += e;
        if constexpr (ENT) r.A = fmaf(e, fmaxf(t, FAR_BELOW), r.A);
    }
}

// Lanes' values, the largest first.  MERGE: the lanes already hold one sequence that falls and then rises, or the other way round.
template <bool MERGE>
__device__ __forceinline__ float sort_lanes(float v) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int k = MERGE ? 32 : 2; k <= 32; k <<= 1) {
#pragma unroll
        for (int j = k >> 1; j > 0; j >>= 1) {
            const float o = __shfl_xor_sync(0xffffffffu, v, j);
            v = ((lane & k) == 0) == ((lane & j) == 0) ? fmaxf(v, o) : fminf(v, o);
        }
    }
    return v;
}

// Numbers that rise as the values do (-0 and 0 are one value).
__device__ __forceinline__ uint32_t ordered(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

constexpr int MOST_TOP = DESLOC_MAX_TOP, CANDIDATES = 1024;

// The part of a row that a block takes, in pieces of 16 bytes: `head` values in front of the first boundary, `pieces`, `tail` values behind.
template <typename T>
struct Part {
    static constexpr int PER = 16 / static_cast<int>(sizeof(T));
    const T *p;
    int head, pieces, tail;
    __device__ __forceinline__ Part(const T *at, int n) : p(at) {
        head = min(n, static_cast<int>((0 - reinterpret_cast<uintptr_t>(at)) & 15u) / static_cast<int>(sizeof(T)));
        pieces = (n - head) / PER;
        tail = n - head - pieces * PER;
    }
    __device__ __forceinline__ int piece_at(int i) const { return head + i * PER; }
    __device__ __forceinline__ int tail_at(int i) const { return head + pieces * PER + i; }
};

// visit(place in the part, value) of all that thread `tid` of `threads` takes, as logprobs_row() took them before.
template <typename T, typename F>
__device__ __forceinline__ void visit_own(const Part<T> &part, int tid, int threads, const F &visit) {
    if (tid < part.head) visit(tid, static_cast<float>(part.p[tid]));
    if (tid < part.tail) visit(part.tail_at(tid), static_cast<float>(part.p[part.tail_at(tid)]));
#pragma unroll 4
    for (int i = tid; i < part.pieces; i += threads) {
        float f[Part<T>::PER];
        load_values(part.p + part.piece_at(i), f);
#pragma unroll
        for (int k = 0; k < Part<T>::PER; ++k) visit(part.piece_at(i) + k, f[k]);
    }
}

template <int THREADS>
struct TopShared {
    float sorted[THREADS / 32][32];
    float value[CANDIDATES];
    int place[CANDIDATES];
    int n;
    float out_value[MOST_TOP];
    int out_place[MOST_TOP];
    unsigned long long best[THREADS / 32];
};

// The candidates' order: larger values first, lower places among equals.  Writes the first `top` of them, -1 where there are fewer.
template <int THREADS>
__device__ __forceinline__ void rank_candidates(TopShared<THREADS> &s, int n, int top) {
    const int tid = threadIdx.x;
    for (int i = tid; i < MOST_TOP; i += THREADS) s.out_value[i] = -INFINITY, s.out_place[i] = -1;
    __syncthreads();
    for (int i = tid; i < n; i += THREADS) {
        const float v = s.value[i];
        const int at = s.place[i];
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += s.value[j] > v || (s.value[j] == v && s.place[j] < at);
        if (rank < top && v > -INFINITY) s.out_value[rank] = v, s.out_place[rank] = at;
    }
    __syncthreads();
}

// The `top` largest values of a part, whatever they are: goes over the part in order and puts what beats the last of the list into it, one at
// a time.  Only for parts with more than CANDIDATES values at or above the line that top_of_part() draws.
template <typename T, int THREADS>
__device__ __noinline__ void top_in_order(const Part<T> part, TopShared<THREADS> &s, int top) {
    const int tid = threadIdx.x;
    for (int i = tid; i < MOST_TOP; i += THREADS) s.out_value[i] = -INFINITY, s.out_place[i] = -1;
    if (tid == 0) s.n = 0;
    __syncthreads();
    const int rounds = 2 + (part.pieces + THREADS - 1) / THREADS;   // the head, the pieces, the tail
    for (int r = 0; r < rounds; ++r) {
        float f[Part<T>::PER];
        int at = 0, have = 0;
        if (r == 0 || r == rounds - 1) {
            if (tid < (r == 0 ? part.head : part.tail)) at = r == 0 ? tid : part.tail_at(tid), f[0] = static_cast<float>(part.p[at]), have = 1;
        } else if ((r - 1) * THREADS + tid < part.pieces) {
            at = part.piece_at((r - 1) * THREADS + tid);
            load_values(part.p + at, f);
            have = Part<T>::PER;
        }
        unsigned left = (1u << have) - 1;
        for (;;) {
            const float line = s.n < top ? -INFINITY : s.out_value[top - 1];
            unsigned long long best = 0;   // value, then low places first
            int which = 0;
#pragma unroll
            for (int k = 0; k < Part<T>::PER; ++k)
                if ((left >> k & 1u) && f[k] > line) {
                    const unsigned long long key = static_cast<unsigned long long>(ordered(f[k])) << 32 | (0xffffffffu - static_cast<unsigned>(at + k));
                    if (key > best) best = key, which = k;
                }
            const unsigned long long own = best;
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) {
                const unsigned long long o = __shfl_xor_sync(0xffffffffu, best, off);
                best = o > best ? o : best;
            }
            if ((tid & 31) == 0) s.best[tid >> 5] = best;
            __syncthreads();
            best = 0;
#pragma unroll
            for (int w = 0; w < THREADS / 32; ++w) best = s.best[w] > best ? s.best[w] : best;
            const int n = s.n;
            __syncthreads();
            if (best == 0) break;
            if (own == best) {   // one thread: places differ
                float v = f[0];
#pragma unroll
                for (int k = 1; k < Part<T>::PER; ++k) v = which == k ? f[k] : v;
                left &= ~(1u << which);
                int i = min(n, top - 1);
                for (; i > 0 && s.out_value[i - 1] < v; --i) s.out_value[i] = s.out_value[i - 1], s.out_place[i] = s.out_place[i - 1];
                s.out_value[i] = v, s.out_place[i] = at + which;
                s.n = min(n + 1, top);
            }
            __syncthreads();
        }
    }
}

// The `top` largest values of a part into s.out_*.  `own`: the largest that this thread has seen (-FLT_MAX: none).  The line is the top-th largest of the
// threads' largest values: at least `top` values lie at or above it (all values, where fewer threads have any), only threads whose largest does have
// such, and these look at what they took once more (some hundred bytes each, from L2).
template <typename T, int THREADS>
__device__ __forceinline__ void top_of_part(const Part<T> &part, TopShared<THREADS> &s, float own, int top) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    s.sorted[warp][lane] = sort_lanes<false>(own);
    if (tid == 0) s.n = 0;
    __syncthreads();
#pragma unroll
    for (int half = THREADS / 64; half > 0; half >>= 1) {
        if (warp < half) s.sorted[warp][lane] = sort_lanes<true>(fmaxf(s.sorted[warp][lane], s.sorted[warp + half][31 - lane]));
        __syncthreads();
    }
    const float line = s.sorted[0][top - 1];
    if (own >= line)
        visit_own(part, tid, THREADS, [&](int at, float x) {
            if (x >= line) {
                const int i = atomicAdd(&s.n, 1);
                if (i < CANDIDATES) s.value[i] = x, s.place[i] = at;
            }
        });
    __syncthreads();
    const int n = s.n;
    if (n <= CANDIDATES) rank_candidates(s, n, top);
    else top_in_order<T, THREADS>(part, s, top);
}

// A block per row, or a cluster of CL blocks that take a part of it each and hand what they found to the first one through its shared
// memory.  Bound: HBM reads of the logits, once; 16-byte loads, four in flight per thread.
template <typename T, bool ENT, bool TOP, int THREADS, int CL>
__device__ __forceinline__ void logprobs_row(const LogprobArgs &a) {
    constexpr int PER = Part<T>::PER, WARPS = THREADS / 32;
    __shared__ Running s_warp[WARPS];
    __shared__ Running s_part[CL];
    __shared__ TopShared<TOP ? THREADS : 32> top;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const unsigned row = blockIdx.x / CL;
    const int rank = static_cast<int>(blockIdx.x % CL);
    begin_and_let_next_begin();
    if constexpr (CL > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");   // (do the blocks exist?  asked below)
    const unsigned i = row / a.inner, j = row - i * a.inner;
    const T *x = static_cast<const T *>(a.x) + i * a.xs0 + j * a.xs1;
    const int per = CL == 1 ? a.vocab : ((a.vocab + CL - 1) / CL + 15) & ~15;
    const int j0 = min(a.vocab, rank * per);
    const Part<T> part(x + j0, min(a.vocab - j0, per));
    wait_for_earlier_kernels();
    int tok = -1;
    float x_tok = 0.f;
    if (tid == 0 && rank == 0) {
        tok = token_at(a.tokens, i * a.tokens.s0 + j * a.tokens.s1, a.vocab);
        if (tok >= 0) x_tok = static_cast<float>(x[tok]);
    }
    Running r{-FLT_MAX, 0.f, 0.f};
    if (tid < part.head) {
        const float f[1] = {static_cast<float>(part.p[tid])};
        take<ENT>(r, f);
    }
    if (tid < part.tail) {
        const float f[1] = {static_cast<float>(part.p[part.tail_at(tid)])};
        take<ENT>(r, f);
    }
    for (int b = tid; b < part.pieces; b += 4 * THREADS) {
        float f[4][PER];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (b + k * THREADS < part.pieces) load_values(part.p + part.piece_at(b + k * THREADS), f[k]);
            else
#pragma unroll
                for (int e = 0; e < PER; ++e) f[k][e] = -INFINITY;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) take<ENT>(r, f[k]);
    }
    const float own = r.m;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        const Running o{__shfl_xor_sync(0xffffffffu, r.m, off), __shfl_xor_sync(0xffffffffu, r.S, off), ENT ? __shfl_xor_sync(0xffffffffu, r.A, off) : 0.f};
        r = lane & off ? join<ENT>(o, r) : join<ENT>(r, o);   // the same order in both lanes
    }
    if (lane == 0) s_warp[warp] = r;
    if constexpr (TOP) top_of_part<T, THREADS>(part, top, own, a.top);   // (its barriers are ours)
    else __syncthreads();
    r = s_warp[0];
#pragma unroll
    for (int w = 1; w < WARPS; ++w) r = join<ENT>(r, s_warp[w]);
    if constexpr (CL > 1) {
        // the parts' sums and [CL][top] candidates go to the first block
        asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
        const auto put = [](void *p, uint32_t v) {
            uint32_t to;
            asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(to) : "r"(smem_u32(p)));
            asm volatile("st.shared::cluster.u32 [%0], %1;" :: "r"(to), "r"(v) : "memory");
        };
        if (tid == 0) {
            put(&s_part[rank].m, __float_as_uint(r.m));
            put(&s_part[rank].S, __float_as_uint(r.S));
            put(&s_part[rank].A, __float_as_uint(r.A));
        }
        if constexpr (TOP) {
            float v = 0.f;
            int at = -1;
            if (tid < a.top) v = top.out_value[tid], at = top.out_place[tid];
            // (every block is done with its own candidates)
            asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
            if (tid < a.top) {
                put(&top.value[rank * a.top + tid], __float_as_uint(v));
                put(&top.place[rank * a.top + tid], static_cast<uint32_t>(j0 + at));
            }
        }
        asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
        if (rank != 0) return;
        r = s_part[0];
#pragma unroll
        for (int k = 1; k < CL; ++k) r = join<ENT>(r, s_part[k]);
        if constexpr (TOP) rank_candidates(top, CL * a.top, a.top);   // (places that hold nothing are -inf, behind all others)
    }
    const float log_sum = logf(r.S);
    const bool empty = r.S == 0.f;
    if (tid == 0) {
        a.lse[row] = empty ? -INFINITY : r.m + log_sum;
        a.logp[row] = tok < 0 ? 0.f : empty ? -INFINITY : (x_tok - r.m) - log_sum;
        if constexpr (ENT) a.entropy[row] = empty ? 0.f : log_sum - LN2 * (r.A / r.S);
    }
    if constexpr (TOP) {
        if (tid < a.top) {
            const float v = top.out_value[tid];
            const bool any = v > -INFINITY;
            a.top_ids[static_cast<long long>(row) * a.top + tid] = any ? top.out_place[tid] : -1;
            a.top_logp[static_cast<long long>(row) * a.top + tid] = any ? (v - r.m) - log_sum : -INFINITY;
        }
    }
}

template <typename T, bool ENT, bool TOP, int THREADS>
__global__ void __launch_bounds__(THREADS) logprobs_kernel(const LogprobArgs a) {
    logprobs_row<T, ENT, TOP, THREADS, 1>(a);
}

constexpr int CLUSTER = 8;

template <typename T, bool ENT, bool TOP, int THREADS>
__global__ void __cluster_dims__(CLUSTER, 1, 1) __launch_bounds__(THREADS) logprobs_cluster_kernel(const LogprobArgs a) {
    logprobs_row<T, ENT, TOP, THREADS, CLUSTER>(a);
}

template <typename T, bool ENT, bool TOP>
cudaError_t launch_rows(const LogprobArgs &a, cudaStream_t stream) {
    // Few long rows: a cluster each.
    if (a.vocab >= 16384 && a.rows <= 148 / CLUSTER * 2)
        return launch_op(logprobs_cluster_kernel<T, ENT, TOP, 512>, dim3(a.rows * CLUSTER), dim3(512), 0, true, stream, a);
    if (a.vocab >= 8192) return launch_op(logprobs_kernel<T, ENT, TOP, 512>, dim3(a.rows), dim3(512), 0, true, stream, a);
    return launch_op(logprobs_kernel<T, ENT, TOP, 128>, dim3(a.rows), dim3(128), 0, true, stream, a);
}

// ---- gradient ----------------------------------------------------------------------------------------
// out_j = a (1[j = token] - p_j) - b p_j (log p_j + H): elementwise over a row.  Bound: HBM, the logits read and as many bytes written.
//
// p_j = exp(x_j - lse) is off by |lse| 2^-24 from the rounding of lse.  Where that is more than an output of the type can bear (1.5e-5 for fp32, a quarter
// of a step for bf16: logits of 1e4, or a row of the type's lowest value), the row's first block takes all of it, and goes over it for the largest
// logit and the sum behind it instead: slow, and rare.
constexpr int GRAD_THREADS = 256, GRAD_AHEAD = 4;

template <typename T>
__device__ __noinline__ Running sum_of_row(const Part<T> part) {
    __shared__ Running s_warp[GRAD_THREADS / 32];
    Running r{-FLT_MAX, 0.f, 0.f};
    visit_own(part, threadIdx.x, GRAD_THREADS, [&](int, float x) {
        const float f[1] = {x};
        take<false>(r, f);
    });
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        const Running o{__shfl_xor_sync(0xffffffffu, r.m, off), __shfl_xor_sync(0xffffffffu, r.S, off), 0.f};
        r = threadIdx.x & off ? join<false>(o, r) : join<false>(r, o);
    }
    if (threadIdx.x % 32 == 0) s_warp[threadIdx.x / 32] = r;
    __syncthreads();
    r = s_warp[0];
#pragma unroll
    for (int w = 1; w < GRAD_THREADS / 32; ++w) r = join<false>(r, s_warp[w]);
    return r;
}

template <typename T, bool ENT>
__global__ void __launch_bounds__(GRAD_THREADS) logprobs_grad_kernel(const LogprobGradArgs a, unsigned blocks) {
    constexpr int PER = Part<T>::PER;
    begin_and_let_next_begin();
    const unsigned row = blockIdx.x / blocks, b = blockIdx.x - row * blocks, i = row / a.inner, j = row - i * a.inner;
    const T *x = static_cast<const T *>(a.x) + i * a.xs0 + j * a.xs1;
    T *out = static_cast<T *>(a.out) + i * a.os0 + j * a.os1;
    // a block's share: whole pieces of 16 bytes of the logits; the first block has what is in front of them, the last one what is behind
    const Part<T> part(x, a.vocab);
    const bool alike = ((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(out)) & 15u) == 0;
    wait_for_earlier_kernels();
    const int tok = token_at(a.tokens, i * a.tokens.s0 + j * a.tokens.s1, a.vocab);
    const float wa = tok < 0 ? 0.f : a.dlogp[row], wb = ENT ? a.dentropy[row] : 0.f;
    const float lse = a.lse[row], H = ENT && wb != 0.f ? a.entropy[row] : 0.f;
    const bool zero = (wa == 0.f && wb == 0.f) || lse == -INFINITY;
    float from = lse, log_sum = 0.f;   // log p = (x - from) - log_sum
    unsigned end = b + 1;              // shares that this block takes: its own, or all of them
    if (fabsf(lse) > (sizeof(T) == 2 ? 16384.f : 256.f) && !zero) {
        if (b != 0) return;
        const Running r = sum_of_row(part);
        from = r.m, log_sum = logf(r.S);
        end = blocks;
        __syncthreads();               // out may be the logits: all of the block have read them
    }
    const auto value = [&](float v, int at) {
        const float lp = (v - from) - log_sum, p = exp2_fast(lp * LOG2E);
        const float w = ENT ? fmaf(wb, fmaxf(lp, FAR_BELOW) + H, wa) : wa;
        const float g = at == tok ? fmaf(-p, w, wa) : -p * w;
        return zero ? 0.f : g;
    };
    for (unsigned share = b; share < end; ++share) {
        const int first = static_cast<int>(share * (GRAD_THREADS * GRAD_AHEAD) + threadIdx.x);
        float f[GRAD_AHEAD][PER];
#pragma unroll
        for (int k = 0; k < GRAD_AHEAD; ++k)
            if (first + k * GRAD_THREADS < part.pieces && !zero) load_values(x + part.piece_at(first + k * GRAD_THREADS), f[k]);
#pragma unroll
        for (int k = 0; k < GRAD_AHEAD; ++k) {
            if (first + k * GRAD_THREADS >= part.pieces) break;
            const int at = part.piece_at(first + k * GRAD_THREADS);
#pragma unroll
            for (int e = 0; e < PER; ++e) f[k][e] = value(f[k][e], at + e);
            if (alike) {
                store_values(out + at, f[k]);
            } else {
#pragma unroll
                for (int e = 0; e < PER; ++e) {
                    const float one[1] = {f[k][e]};
                    store_values(out + at + e, one);
                }
            }
        }
    }
    const int edge = static_cast<int>(threadIdx.x);
    const int at = b == 0 && edge < part.head ? edge : end == blocks && edge >= 32 && edge - 32 < part.tail ? part.tail_at(edge - 32) : -1;
    if (at >= 0) {
        const float one[1] = {value(zero ? 0.f : static_cast<float>(x[at]), at)};
        store_values(out + at, one);
    }
}

template <typename T, bool ENT>
cudaError_t launch_grad(const LogprobGradArgs &a, cudaStream_t stream) {
    constexpr int SHARE = GRAD_THREADS * GRAD_AHEAD * Part<T>::PER;
    const unsigned blocks = static_cast<unsigned>((static_cast<int64_t>(a.vocab) + SHARE - 1) / SHARE);
    if (static_cast<int64_t>(blocks) * a.rows > 0x7fffffffLL) return cudaErrorInvalidConfiguration;   // (beyond any memory)
    return launch_op(logprobs_grad_kernel<T, ENT>, dim3(blocks * a.rows), dim3(GRAD_THREADS), 0, true, stream, a, blocks);
}

}  // namespace

cudaError_t launch_logprobs(const LogprobArgs &a, bool bf16, cudaStream_t stream) {
    using bf = __nv_bfloat16;
    if (a.top > 0)
        return bf16 ? (a.entropy ? launch_rows<bf, true, true> : launch_rows<bf, false, true>)(a, stream)
                    : (a.entropy ? launch_rows<float, true, true> : launch_rows<float, false, true>)(a, stream);
    return bf16 ? (a.entropy ? launch_rows<bf, true, false> : launch_rows<bf, false, false>)(a, stream)
                : (a.entropy ? launch_rows<float, true, false> : launch_rows<float, false, false>)(a, stream);
}

cudaError_t launch_logprobs_grad(const LogprobGradArgs &a, bool bf16, cudaStream_t stream) {
    using bf = __nv_bfloat16;
    return bf16 ? (a.dentropy ? launch_grad<bf, true> : launch_grad<bf, false>)(a, stream)
                : (a.dentropy ? launch_grad<float, true> : launch_grad<float, false>)(a, stream);
}

}  // namespace desloc

namespace {

// Checks of rows that both calls make.
int check_rows(int64_t outer, int64_t inner, int64_t vocab, const desloc_rows *logits, const desloc_rows *tokens, int cuda_device) {
    if (!logits || !tokens) return DESLOC_E_NULL;
    if (outer < 0 || inner < 0 || vocab < 1 || vocab > (1 << 30) || cuda_device < 0) return DESLOC_E_RANGE;
    if (outer > 0 && inner > (1 << 28) / outer) return DESLOC_E_RANGE;
    return desloc::is_value_rows(*logits) && desloc::is_token_rows(*tokens) ? DESLOC_OK : DESLOC_E_INVALID;
}

// Runs `call` with the device current.
template <typename F>
int on_device(int device, const F &call) {
    int before = -1;
    cudaError_t e = cudaGetDevice(&before);
    if (e == cudaSuccess && before != device) e = cudaSetDevice(device);
    if (e == cudaSuccess) e = call();
    if (before >= 0 && before != device) cudaSetDevice(before);
    if (e == cudaSuccess) return DESLOC_OK;
    (void)cudaGetLastError();
    return DESLOC_E_CUDA;
}

}  // namespace

extern "C" {

int desloc_token_logprobs(int64_t outer, int64_t inner, int64_t vocab, const desloc_rows *logits, const desloc_rows *tokens, int32_t top,
                          float *logp, float *lse, float *entropy, int64_t *top_ids, float *top_logp, int cuda_device, void *stream) {
    desloc::NvtxRange range("desloc_token_logprobs");
    const int rc = check_rows(outer, inner, vocab, logits, tokens, cuda_device);
    if (rc != DESLOC_OK) return rc;
    if (top < 0 || top > DESLOC_MAX_TOP) return DESLOC_E_RANGE;
    if (outer * inner == 0) return DESLOC_OK;
    if (!logits->data || !tokens->data || !logp || !lse || (top > 0 && (!top_ids || !top_logp))) return DESLOC_E_NULL;
    desloc::LogprobArgs a{};
    a.x = logits->data;
    a.xs0 = logits->stride[0], a.xs1 = logits->stride[1];
    a.tokens = desloc::token_rows(*tokens);
    a.rows = static_cast<unsigned>(outer * inner), a.inner = static_cast<unsigned>(inner);
    a.vocab = static_cast<int>(vocab), a.top = top;
    a.logp = logp, a.lse = lse, a.entropy = entropy;
    a.top_ids = reinterpret_cast<long long *>(top_ids), a.top_logp = top_logp;
    return on_device(cuda_device, [&] { return desloc::launch_logprobs(a, logits->dtype == DESLOC_BF16, static_cast<cudaStream_t>(stream)); });
}

int desloc_token_logprobs_grad(int64_t outer, int64_t inner, int64_t vocab, const desloc_rows *logits, const desloc_rows *tokens,
                               const float *lse, const float *dlogp, const float *entropy, const float *dentropy, const desloc_rows *out,
                               int cuda_device, void *stream) {
    desloc::NvtxRange range("desloc_token_logprobs_grad");
    const int rc = check_rows(outer, inner, vocab, logits, tokens, cuda_device);
    if (rc != DESLOC_OK) return rc;
    if (!out) return DESLOC_E_NULL;
    if (!desloc::is_value_rows(*out) || out->dtype != logits->dtype) return DESLOC_E_INVALID;
    if (outer * inner == 0) return DESLOC_OK;
    if (!logits->data || !tokens->data || !out->data || !lse || !dlogp || (dentropy && !entropy)) return DESLOC_E_NULL;
    desloc::LogprobGradArgs a{};
    a.x = logits->data;
    a.xs0 = logits->stride[0], a.xs1 = logits->stride[1];
    a.tokens = desloc::token_rows(*tokens);
    a.rows = static_cast<unsigned>(outer * inner), a.inner = static_cast<unsigned>(inner);
    a.vocab = static_cast<int>(vocab);
    a.lse = lse, a.dlogp = dlogp, a.entropy = entropy, a.dentropy = dentropy;
    a.out = out->data;
    a.os0 = out->stride[0], a.os1 = out->stride[1];
    return on_device(cuda_device, [&] { return desloc::launch_logprobs_grad(a, logits->dtype == DESLOC_BF16, static_cast<cudaStream_t>(stream)); });
}

}  // extern "C"
