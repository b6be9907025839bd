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

// Running softmax of a part of a row: largest value m, S = sum of 2^t and A = sum of t 2^t, with t = x log2 e - base(m), one rounding: the
// rounding of base(m) = m log2 e is the same in every term, and log_sum_of() takes it out again.  Rows whose largest value is beyond HUGE_LOGIT, where that
// rounding is no small exponent, have t = (x - m) log2 e.  Parts without values (or of nothing but -inf) have m = -FLT_MAX and S = 0; NaN and +inf end in a NaN S.
struct Running {
    float m, S, A;
};
constexpr float HUGE_LOGIT = 1e6f;
__device__ __forceinline__ float base_of(float m) { return __fmul_rn(m, LOG2E); }
__device__ __forceinline__ bool is_huge(float m) { return fabsf(m) > HUGE_LOGIT; }
__device__ __forceinline__ float behind_base(float m) { return fmaf(m, LOG2E, -base_of(m)); }   // what the rounding took

template <bool ENT>
__device__ __forceinline__ void raise_to(Running &r, float m) {
    float d = base_of(r.m) - base_of(m);
    if (is_huge(r.m) || is_huge(m)) d = is_huge(r.m) && is_huge(m) ? (r.m - m) * LOG2E : is_huge(m) ? d - behind_base(m) : d + behind_base(r.m);
    d = fmaxf(d, FAR_BELOW);   // (NaN, of infinities, too)
    const float f = exp2_fast(d);
    if constexpr (ENT) r.A = f * fmaf(r.S, d, r.A);
    r.S *= f;
    r.m = m;
}

// The lanes' sums as one, in all of them: of groups of LANES.
template <bool ENT, int LANES>
__device__ __forceinline__ Running join_lanes(Running r) {
    float m = r.m;
#pragma unroll
    for (int off = LANES / 2; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, off));
    raise_to<ENT>(r, m);
#pragma unroll
    for (int off = LANES / 2; off > 0; off >>= 1) {
        r.S += __shfl_xor_sync(0xffffffffu, r.S, off);
        if constexpr (ENT) r.A += __shfl_xor_sync(0xffffffffu, r.A, off);
    }
    return r;
}

// One value.
template <bool ENT>
__device__ __forceinline__ void take(Running &r, float x) {
    if (x > r.m) raise_to<ENT>(r, x);
    const float t = is_huge(r.m) ? (x - r.m) * LOG2E : fmaf(x, LOG2E, -base_of(r.m)), e = exp2_fast(t);
    r.S += e;
    if constexpr (ENT) r.A = fmaf(e, fmaxf(t, FAR_BELOW), r.A);
}

// log sum exp(x - m).
__device__ __forceinline__ float log_sum_of(const Running &r) {
    const float l = logf(r.S);
    return is_huge(r.m) ? l : l - LN2 * behind_base(r.m);
}

// Sixteen bytes of a row as values; the largest of several; what stands in the place of missing ones.
template <typename T>
struct Words;
template <>
struct Words<float> {
    static constexpr uint32_t NONE = 0xff800000u;   // -inf
    static __device__ __forceinline__ float2 pair(const uint4 &w, int k) {
        return k == 0 ? make_float2(__uint_as_float(w.x), __uint_as_float(w.y)) : make_float2(__uint_as_float(w.z), __uint_as_float(w.w));
    }
    template <int N>
    static __device__ __forceinline__ float largest(const uint4 (&w)[N]) {
        float m = -INFINITY;
#pragma unroll
        for (int k = 0; k < N; ++k)
            m = fmaxf(m, fmaxf(fmaxf(__uint_as_float(w[k].x), __uint_as_float(w[k].y)), fmaxf(__uint_as_float(w[k].z), __uint_as_float(w[k].w))));
        return m;
    }
    static constexpr uint32_t LOWEST = 0xfcf0bdc2u;   // -1e37: finite, and its exponential 0
    static __device__ __forceinline__ uint32_t both(float x) { return __float_as_uint(x); }
    // The larger of each; NaN stays.
    static __device__ __forceinline__ uint32_t at_least(uint32_t low, uint32_t w) {
        float r;
        asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(__uint_as_float(w)), "f"(__uint_as_float(low)));
        return __float_as_uint(r);
    }
};
template <>
struct Words<__nv_bfloat16> {
    static constexpr uint32_t NONE = 0xff80ff80u;
    static __device__ __forceinline__ float2 pair(const uint4 &w, int k) {
        const uint32_t v = k == 0 ? w.x : k == 1 ? w.y : k == 2 ? w.z : w.w;
        return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
    }
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
        uint32_t r;
        asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    template <int N>
    static __device__ __forceinline__ float largest(const uint4 (&w)[N]) {
        uint32_t m = NONE;
#pragma unroll
        for (int k = 0; k < N; ++k) m = larger(m, larger(larger(w[k].x, w[k].y), larger(w[k].z, w[k].w)));
        return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
    }
    static constexpr uint32_t LOWEST = 0xfcf0fcf0u;
    static __device__ __forceinline__ uint32_t both(float x) { return pack_bf16(x, x); }
    static __device__ __forceinline__ uint32_t at_least(uint32_t low, uint32_t w) {
        uint32_t r;
        asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(w), "r"(low));
        return r;
    }
};

template <typename T>
__device__ __forceinline__ void raise_words(uint32_t low, uint4 &w) {
    w = make_uint4(Words<T>::at_least(low, w.x), Words<T>::at_least(low, w.y), Words<T>::at_least(low, w.z), Words<T>::at_least(low, w.w));
}

// A piece, value by value: of rows with values beyond HUGE_LOGIT only.
template <typename T, bool ENT>
__device__ __noinline__ Running take_slowly(Running r, uint4 w) {
#pragma unroll
    for (int e = 0; e < 8 / static_cast<int>(sizeof(T)); ++e) {
        const float2 x = Words<T>::pair(w, e);
        take<ENT>(r, x.x);
        take<ENT>(r, x.y);
    }
    return r;
}

// N pieces, two values per instruction.
template <typename T, bool ENT, int N>
__device__ __forceinline__ void take_pieces(Running &r, uint4 (&w)[N]) {
    const float top = Words<T>::largest(w);
    if (top > r.m) raise_to<ENT>(r, top);
    if (is_huge(r.m)) {
#pragma unroll
        for (int k = 0; k < N; ++k) r = take_slowly<T, ENT>(r, w[k]);
        return;
    }
    const float b = base_of(r.m);
    const float2 scale = make_float2(LOG2E, LOG2E), from = make_float2(-b, -b);
    float2 S = make_float2(r.S, 0.f), A = make_float2(ENT ? r.A : 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < N; ++k) {
        if constexpr (ENT) raise_words<T>(Words<T>::LOWEST, w[k]);
#pragma unroll
        for (int e = 0; e < 8 / static_cast<int>(sizeof(T)); ++e) {
            const float2 t = __ffma2_rn(Words<T>::pair(w[k], e), scale, from), p = make_float2(exp2_fast(t.x), exp2_fast(t.y));
            S = __fadd2_rn(S, p);
            if constexpr (ENT) A = __ffma2_rn(p, t, A);
        }
    }
    r.S = S.x + S.y;
    if constexpr (ENT) r.A = A.x + A.y;
}

// Lanes' values, the largest first.  MERGE: they fall and then rise, or the other way round, already.
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

// A value and its place as one number: larger for larger values (-0 and 0 are one), then for lower places; 0 for nothing.
using Key = unsigned long long;
__device__ __forceinline__ Key key_of(float x, int place) {
    const uint32_t b = __float_as_uint(x + 0.f);
    return static_cast<Key>(b & 0x80000000u ? ~b : b | 0x80000000u) << 32 | (0xffffffffu - static_cast<uint32_t>(place));
}
__device__ __forceinline__ int place_of(Key key) { return static_cast<int>(0xffffffffu - static_cast<uint32_t>(key)); }
__device__ __forceinline__ float value_of(Key key) {
    const uint32_t b = static_cast<uint32_t>(key >> 32);
    return __uint_as_float(b & 0x80000000u ? b ^ 0x80000000u : ~b);
}

constexpr int MOST_TOP = DESLOC_MAX_TOP, WARP_ROWS = 4;
__host__ __device__ constexpr int candidates(int threads) { return threads > 32 ? 1024 : 256; }   // that a block has room for

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

// visit(place in the part, value) of all that thread `tid` of THREADS takes in logprobs_row(), lane `lane` of `lanes` that share them.
template <int THREADS, typename T, typename F>
__device__ __forceinline__ void visit_own(const Part<T> &part, int tid, int lane, int lanes, const F &visit) {
    if (lane == 0 && tid < part.head) visit(tid, static_cast<float>(part.p[tid]));
    if (lane == 0 && tid < part.tail) visit(part.tail_at(tid), static_cast<float>(part.p[part.tail_at(tid)]));
#pragma unroll 4
    for (long long i = tid + lane * THREADS; i < part.pieces; i += lanes * THREADS) {
        const int at = part.piece_at(static_cast<int>(i));
        float f[Part<T>::PER];
        load_values(part.p + at, f);
#pragma unroll
        for (int k = 0; k < Part<T>::PER; ++k) visit(at + k, f[k]);
    }
}

// A barrier of the threads that share a row.
template <int THREADS>
__device__ __forceinline__ void row_barrier() {
    if constexpr (THREADS == 32) __syncwarp();
    else __syncthreads();
}

template <int THREADS>
struct TopShared {
    float own[THREADS / 32][32];
    float line;
    int n;
    Key key[candidates(THREADS)];
    Key out[MOST_TOP];   // the largest ones, in order, where they have been ranked
    Key best[THREADS / 32];
};

// put(rank, key) for the `top` largest of n keys, in order, and put(rank, 0) where there are fewer.  (Keys but 0 differ.)
template <int THREADS, typename Put>
__device__ __forceinline__ void rank_keys(const Key *keys, int n, int top, const Put &put) {
    for (int i = threadIdx.x; i < max(n, top); i += THREADS) {
        const Key own = i < n ? keys[i] : 0;
        int rank = 0, real = 0;
#pragma unroll 8
        for (int j = 0; j < n; ++j) {
            const Key k = keys[j];
            rank += k > own;
            real += k != 0;
        }
        if (own != 0 && rank < top) put(rank, own);
        if (i >= real && i < top) put(i, Key{0});
    }
}

// The `top` largest values of a part, whatever they are, into s.out: goes over the part in order and puts what beats the last of the list into it,
// one at a time.  Only for parts with more than candidates(THREADS) values at or above the line that candidates_of_part() draws.
template <typename T, int THREADS>
__device__ __noinline__ void top_in_order(const Part<T> part, TopShared<THREADS> &s, int top) {
    const int tid = threadIdx.x;
    for (int i = tid; i < MOST_TOP; i += THREADS) s.out[i] = 0;
    row_barrier<THREADS>();
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
            const Key line = s.out[top - 1];
            Key own = 0;
            int which = 0;
#pragma unroll
            for (int k = 0; k < Part<T>::PER; ++k)
                if ((left >> k & 1u) && f[k] > -INFINITY) {
                    const Key key = key_of(f[k], at + k);
                    if (key > line && key > own) own = key, which = k;
                }
            Key best = own;
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) {
                const Key o = __shfl_xor_sync(0xffffffffu, best, off);
                best = o > best ? o : best;
            }
            if ((tid & 31) == 0) s.best[tid >> 5] = best;
            row_barrier<THREADS>();
            best = 0;
#pragma unroll
            for (int w = 0; w < THREADS / 32; ++w) best = s.best[w] > best ? s.best[w] : best;
            if (best == 0) break;   // (in all threads)
            if (own == best) {      // one thread: places differ
                left &= ~(1u << which);
                int i = top - 1;
                for (; i > 0 && s.out[i - 1] < own; --i) s.out[i] = s.out[i - 1];
                s.out[i] = own;
            }
            row_barrier<THREADS>();
        }
        row_barrier<THREADS>();   // s.best has been read
    }
}

// Candidates for the `top` largest values of a part into s.key; how many, which may be more than there is room for.  s.own holds the largest
// that each thread has seen (-FLT_MAX: none), behind a barrier.  The line is the top-th largest of the threads' largest values, or of 32 groups' of threads where that
// is near enough (32 groups and 32 alternatives: the line is the least of all, and half of the row above it; 16384 rows of 1000 bf16 logits 66 us and 168): at
// least `top` values lie at or above it (all values, where fewer have any), only threads whose largest does have such, and their warps look at what these
// took once more (some hundred bytes each, from L2).
constexpr int TOP_OF_GROUPS = 16;

template <typename T, int THREADS>
__device__ __forceinline__ int candidates_of_part(const Part<T> &part, TopShared<THREADS> &s, float own, int top) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (THREADS == 32 || top <= TOP_OF_GROUPS) {
        if (warp == 0) {
            float m = s.own[0][lane];
#pragma unroll
            for (int w = 1; w < THREADS / 32; ++w) m = fmaxf(m, s.own[w][lane]);
            m = sort_lanes<false>(m);
            if (lane == top - 1) s.line = m;
        }
    } else {
        s.own[warp][lane] = sort_lanes<false>(own);
        row_barrier<THREADS>();
#pragma unroll
        for (int half = THREADS / 64; half > 0; half >>= 1) {
            if (warp < half) {
                const float m = sort_lanes<true>(fmaxf(s.own[warp][lane], s.own[warp + half][31 - lane]));
                s.own[warp][lane] = m;
                if (half == 1 && lane == top - 1) s.line = m;
            }
            if (half > 1) row_barrier<THREADS>();
        }
    }
    if (tid == 0) s.n = 0;
    row_barrier<THREADS>();
    const float line = s.line;
    const auto collect = [&](int at, float x) {
        if (x >= line) {
            const int i = atomicAdd(&s.n, 1);
            if (i < candidates(THREADS)) s.key[i] = key_of(x, at);
        }
    };
    // (a few pieces each: every thread its own, all at once)
    if (part.pieces <= 4 * THREADS) {
        if (own >= line) visit_own<THREADS>(part, tid, 0, 1, collect);
    } else {
        for (unsigned who = __ballot_sync(0xffffffffu, own >= line); who; who &= who - 1)
            visit_own<THREADS>(part, (tid & ~31) + __ffs(who) - 1, tid & 31, 32, collect);
    }
    row_barrier<THREADS>();
    return s.n;
}

// A block per row, or a cluster of CL blocks that take a part of it each and hand what they found to the first one through its shared
// memory.  Bound: HBM reads of the logits, once (16-byte loads, four to eight in flight per thread), then the exponentials, 16 per clock and SM.
// 4096 rows of 49152 bf16 logits with entropy and five alternatives: 83 us, 4.9 TB/s (0.74 of copy), 76 at its best.  Before, each at its best: value by
// value, blocks of 512 threads, the alternatives looked for by single threads 172; blocks of 256 127 (of 128 134); two values per instruction and warps that
// look for alternatives 82; whole rounds of loads without conditions and five blocks per SM 78 (four 82).  Without alternatives 6 us less.
// Four rows of 49152 with 20 alternatives, clusters: 10.5 to 11.5 us (before keys that are ranked in one pass, and one barrier more, 23.7).
template <typename T, bool ENT, bool TOP, int THREADS, int CL>
__device__ __forceinline__ void logprobs_row(const LogprobArgs &a) {
    constexpr int WARPS = THREADS / 32, AHEAD = 4;
    constexpr int ROWS = THREADS == 32 ? WARP_ROWS : 1;   // of a block: rows of a warp each share one
    __shared__ Running s_warps[ROWS][WARPS];
    __shared__ Running s_part[CL];
    __shared__ TopShared<THREADS> tops[TOP ? ROWS : 1];
    __shared__ Key s_lists[TOP && CL > 1 ? CL * MOST_TOP : 1];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const unsigned slot = ROWS > 1 ? threadIdx.y : 0, row = blockIdx.x / CL * ROWS + slot;
    const int rank = static_cast<int>(blockIdx.x % CL);
    Running(&s_warp)[WARPS] = s_warps[slot];
    auto &top = tops[TOP ? slot : 0];
    begin_and_let_next_begin();
    if (ROWS > 1 && row >= a.rows) {
        wait_for_earlier_kernels();
        return;
    }
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
    const uint4 *const pieces = reinterpret_cast<const uint4 *>(part.p + part.head);
    // whole rounds of AHEAD pieces per thread, then what is left; the next round's loads are on their way meanwhile
    const int rounds = part.pieces / (AHEAD * THREADS);
    uint4 next[AHEAD];
    const auto load = [&](int round) {
        const uint4 *const p = pieces + static_cast<long long>(round) * (AHEAD * THREADS) + tid;
        const int left = part.pieces - round * (AHEAD * THREADS) - tid;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            constexpr uint32_t none = Words<T>::NONE;
            if (round < rounds) next[k] = p[k * THREADS];
            else next[k] = k * THREADS < left ? p[k * THREADS] : make_uint4(none, none, none, none);
        }
    };
    load(0);
    if (tid < part.head) take<ENT>(r, static_cast<float>(part.p[tid]));
    if (tid < part.tail) take<ENT>(r, static_cast<float>(part.p[part.tail_at(tid)]));
    for (int round = 0; round < rounds; ++round) {
        uint4 w[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) w[k] = next[k];
        load(round + 1);
        take_pieces<T, ENT>(r, w);
    }
    if (rounds * (AHEAD * THREADS) + tid < part.pieces) take_pieces<T, ENT>(r, next);
    const float own = r.m;
    if constexpr (TOP) top.own[warp][lane] = own;
    r = join_lanes<ENT, 32>(r);
    if (lane == 0) s_warp[warp] = r;
    row_barrier<THREADS>();
    int found = 0;
    if constexpr (TOP) {
        found = candidates_of_part(part, top, own, a.top);
        if (found > candidates(THREADS)) top_in_order<T, THREADS>(part, top, a.top);
    }
    const bool listed = found > candidates(THREADS);   // they are in top.out, in order, not among the candidates
    if (CL == 1 && warp * 32 >= (listed ? 1 : max(found, 1))) return;
    r = join_lanes<ENT, WARPS>(s_warp[lane % WARPS]);
    const Key *keys = listed ? top.out : top.key;
    int n = listed ? a.top : found;
    if constexpr (CL > 1) {
        // the parts' sums and lists go to the first block
        asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
        const auto there = [](void *p) {
            uint32_t to;
            asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(to) : "r"(smem_u32(p)));
            return to;
        };
        const auto put = [&](void *p, uint32_t v) { asm volatile("st.shared::cluster.u32 [%0], %1;" :: "r"(there(p)), "r"(v) : "memory"); };
        if (tid == 0) {
            put(&s_part[rank].m, __float_as_uint(r.m));
            put(&s_part[rank].S, __float_as_uint(r.S));
            put(&s_part[rank].A, __float_as_uint(r.A));
        }
        if constexpr (TOP)
            rank_keys<THREADS>(keys, n, a.top, [&](int k, Key key) {
                const Key moved = key ? key - static_cast<Key>(j0) : 0;   // (the place in the row)
                asm volatile("st.shared::cluster.u64 [%0], %1;" :: "r"(there(&s_lists[rank * a.top + k])), "l"(moved) : "memory");
            });
        asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
        if (rank != 0) return;
        r = join_lanes<ENT, CL>(s_part[lane % CL]);
        keys = s_lists, n = CL * a.top;
    }
    const float log_sum = log_sum_of(r);
    const bool empty = r.S == 0.f;
    if (tid == 0) {
        a.lse[row] = empty ? -INFINITY : r.m + log_sum;
        a.logp[row] = tok < 0 ? 0.f : empty ? -INFINITY : (x_tok - r.m) - log_sum;
        if constexpr (ENT) a.entropy[row] = empty ? 0.f : logf(r.S) - LN2 * (r.A / r.S);
    }
    if constexpr (TOP)
        rank_keys<THREADS>(keys, n, a.top, [&](int k, Key key) {
            a.top_ids[static_cast<long long>(row) * a.top + k] = key ? place_of(key) : -1;
            a.top_logp[static_cast<long long>(row) * a.top + k] = key ? (value_of(key) - r.m) - log_sum : -INFINITY;
        });
}

template <typename T, bool ENT, bool TOP, int THREADS>
__global__ void __launch_bounds__(THREADS > 32 ? THREADS : 32 * WARP_ROWS, THREADS > 32 ? 1280 / THREADS : 10) logprobs_kernel(const LogprobArgs a) {
    logprobs_row<T, ENT, TOP, THREADS, 1>(a);
}

constexpr int CLUSTER = 8;

template <typename T, bool ENT, bool TOP, int THREADS>
__global__ void __cluster_dims__(CLUSTER, 1, 1) __launch_bounds__(THREADS) logprobs_cluster_kernel(const LogprobArgs a) {
    logprobs_row<T, ENT, TOP, THREADS, CLUSTER>(a);
}

template <typename T, bool ENT, bool TOP>
cudaError_t launch_rows(const LogprobArgs &a, cudaStream_t stream) {
    // Few long rows: a cluster each.  Shorter ones: as many threads as have a few pieces each.
    if (a.vocab >= 16384 && a.rows <= 148 / CLUSTER * 2)
        return launch_op(logprobs_cluster_kernel<T, ENT, TOP, 256>, dim3(a.rows * CLUSTER), dim3(256), 0, true, stream, a);
    // 16384 rows of 1000 bf16 logits: a warp each, four to a block, 10.5 us (one to a block 18.8), 128 threads 27.2, 256 45.3; 7500 of 20000 with five
    // alternatives 85, 67, 83; 1024 of 33000 33, 23, 20.  (More alternatives than 32 groups tell apart: 128 threads at least.)
    constexpr int FEW = 1024, MANY = 4096;
    const int pieces = TOP && a.top > TOP_OF_GROUPS && a.vocab / Part<T>::PER < FEW ? FEW : a.vocab / Part<T>::PER;
    if (pieces >= MANY) return launch_op(logprobs_kernel<T, ENT, TOP, 256>, dim3(a.rows), dim3(256), 0, true, stream, a);
    if (pieces >= FEW) return launch_op(logprobs_kernel<T, ENT, TOP, 128>, dim3(a.rows), dim3(128), 0, true, stream, a);
    return launch_op(logprobs_kernel<T, ENT, TOP, 32>, dim3((a.rows + WARP_ROWS - 1) / WARP_ROWS), dim3(32, WARP_ROWS), 0, true, stream, a);
}

// ---- gradient ----------------------------------------------------------------------------------------
// out_j = a (1[j = token] - p_j) - b p_j (log p_j + H): elementwise over a row.  Bound: HBM, the logits read and as many bytes written.
// 4096 rows of 49152 bf16 logits: 122 us, 6.6 TB/s (1.01 of copy); value by value 169; shares of 2 and 8 pieces a thread instead of 4 143 and 122.
//
// p_j = exp(x_j - lse) is off by |lse| 2^-24 of itself from the rounding of lse, and what the token's own entry and the entropy's part leave of a difference
// is off by as much of p, however little is left.  Where that passes 1.5e-5 (FAR_LSE; a few steps of 1 - p already in bf16, where the next logit is 8 below),
// the row's first block takes all of the row, and goes over it for the largest logit and the sum behind it instead: slow (4096 rows of 49152 bf16 logits at
// 300: 502 us instead of 119, fp32 669 instead of 233), and rare.
constexpr int GRAD_THREADS = 256, GRAD_AHEAD = 4;

// With entropy, log p is a factor beside the caller's weight.  Logits more than NO_LOGIT below lse, whose p is 0 (2^-126 is e^-87; bf16's steps at the largest
// lse take one of the 200), stand NO_LOGIT below it, so that 0 * weight * log p is 0 for weights up to MOST_WEIGHT; rows with larger ones go value by value.
constexpr float NO_LOGIT = 200.f, MOST_WEIGHT = 1e30f, FAR_LSE = 256.f;

template <typename T>
__device__ __noinline__ Running sum_of_row(const Part<T> part) {
    __shared__ Running s_warp[GRAD_THREADS / 32];
    Running r{-FLT_MAX, 0.f, 0.f};
    visit_own<GRAD_THREADS>(part, threadIdx.x, 0, 1, [&](int, float x) { take<false>(r, x); });
    r = join_lanes<false, 32>(r);
    if (threadIdx.x % 32 == 0) s_warp[threadIdx.x / 32] = r;
    __syncthreads();
    return join_lanes<false, GRAD_THREADS / 32>(s_warp[threadIdx.x % (GRAD_THREADS / 32)]);
}

// All of a row with a large lse or weights that a product with log p may not bear, value by value.
template <typename T, bool ENT>
__device__ __noinline__ void grad_slowly(const Part<T> part, T *out, int tok, float wa, float wb, float H) {
    const Running r = sum_of_row(part);
    const float log_sum = log_sum_of(r);
    __syncthreads();   // out may be the logits: all of the block have read them
    const int n = part.head + part.pieces * Part<T>::PER + part.tail;
    for (int j = threadIdx.x; j < n; j += GRAD_THREADS) {
        const float lp = (static_cast<float>(part.p[j]) - r.m) - log_sum, p = exp2_fast(lp * LOG2E), one = j == tok ? -expm1f(lp) * wa : -p * wa;
        const float g[1] = {ENT ? fmaf(-p * (fmaxf(lp, FAR_BELOW) + H), wb, one) : one};   // (0 comes before the weight)
        store_values(out + j, g);
    }
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
    const uint4 *const pieces = reinterpret_cast<const uint4 *>(x + part.head);
    const int first = static_cast<int>(b * (GRAD_THREADS * GRAD_AHEAD) + threadIdx.x), edge = static_cast<int>(threadIdx.x);
    const int edge_at = b == 0 && edge < part.head ? edge : b == blocks - 1 && edge >= 32 && edge - 32 < part.tail ? part.tail_at(edge - 32) : -1;
    wait_for_earlier_kernels();
    const int tok = token_at(a.tokens, i * a.tokens.s0 + j * a.tokens.s1, a.vocab);
    const float wa = tok < 0 ? 0.f : a.dlogp[row], wb = ENT ? a.dentropy[row] : 0.f;
    const float lse = a.lse[row], H = ENT && wb != 0.f ? a.entropy[row] : 0.f;
    if ((wa == 0.f && wb == 0.f) || lse == -INFINITY) {
        const float none[PER] = {};
#pragma unroll
        for (int k = 0; k < GRAD_AHEAD; ++k) {
            const int at = part.piece_at(first + k * GRAD_THREADS);
            if (first + k * GRAD_THREADS >= part.pieces) break;
            if (alike) store_values(out + at, none);
            else
#pragma unroll
                for (int e = 0; e < PER; ++e) out[at + e] = T(0.f);
        }
        if (edge_at >= 0) out[edge_at] = T(0.f);
        return;
    }
    if (fabsf(lse) > FAR_LSE || fabsf(wa) > MOST_WEIGHT || (ENT && fabsf(wb) > MOST_WEIGHT)) {
        if (b == 0) grad_slowly<T, ENT>(part, out, tok, wa, wb, H);
        return;
    }
    // p = 2^t / 2^off with t = x log2 e - base, base = lse log2 e rounded and off what the rounding took; -w = c0 + c1 t
    const float base = base_of(lse), off = behind_base(lse), q = exp2_fast(-off);
    const float c1 = ENT ? -q * wb * LN2 : 0.f, c0 = -q * (ENT ? fmaf(wb, H - off * LN2, wa) : wa);
    const float2 scale = make_float2(LOG2E, LOG2E), from = make_float2(-base, -base), C0 = make_float2(c0, c0), C1 = make_float2(c1, c1);
    const uint32_t low = Words<T>::both(lse - NO_LOGIT);
    uint4 w[GRAD_AHEAD];
#pragma unroll
    for (int k = 0; k < GRAD_AHEAD; ++k)
        if (first + k * GRAD_THREADS < part.pieces) w[k] = pieces[first + k * GRAD_THREADS];
#pragma unroll
    for (int k = 0; k < GRAD_AHEAD; ++k) {
        if (first + k * GRAD_THREADS >= part.pieces) break;
        const int at = part.piece_at(first + k * GRAD_THREADS);
        if constexpr (ENT) raise_words<T>(low, w[k]);
        float g[PER];
#pragma unroll
        for (int e = 0; e < PER / 2; ++e) {
            const float2 t = __ffma2_rn(Words<T>::pair(w[k], e), scale, from), p = make_float2(exp2_fast(t.x), exp2_fast(t.y));
            const float2 v = __fmul2_rn(p, ENT ? __ffma2_rn(t, C1, C0) : C0);
            g[2 * e] = v.x, g[2 * e + 1] = v.y;
        }
        if (static_cast<unsigned>(tok - at) < PER)
#pragma unroll
            for (int e = 0; e < PER; ++e) g[e] += tok == at + e ? wa : 0.f;
        if (alike) {
            store_values(out + at, g);
        } else {
#pragma unroll
            for (int e = 0; e < PER; ++e) {
                const float one[1] = {g[e]};
                store_values(out + at + e, one);
            }
        }
    }
    if (edge_at >= 0) {
        float t = fmaf(static_cast<float>(x[edge_at]), LOG2E, -base);
        const float p = exp2_fast(t);
        if constexpr (ENT) t = fmaxf(t, -NO_LOGIT * LOG2E);
        const float g[1] = {p * (ENT ? fmaf(t, c1, c0) : c0) + (edge_at == tok ? wa : 0.f)};
        store_values(out + edge_at, g);
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
    if (desloc::rows_overlap(*out, outer, inner, vocab)) return DESLOC_E_INVALID;
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
