// Orthogonalised updates of small matrices: a block takes one from the momentum to the result, nothing in between leaves the SM.
#include "desloc_blocks.cuh"
#include "desloc_gemm.cuh"

#include <cstring>
#include <type_traits>

namespace desloc {

namespace {

// X, the shorter side as rows (tall matrices are turned as they come), G and then the polynomial P of G lie in shared memory as operands of the tensor cores, in blocks of 64
// columns (128 bytes, swizzled).  The same bytes of X serve both products: rows of k for G = X X^T, columns of n for P X.  Every value is two fp16 numbers, hi + lo, and a
// product is three, hi hi + hi lo + lo hi: 20 bits, at no cost that shows here.  What takes time is latency: three products, each behind the other, a step, with all threads
// turning sums into operands in between.  Two 72 x 72 matrices 28 us (92 in the seventeen launches of the kernels for large ones), 3.6 of it a step; 56 of up to 200 x 72 as a step of x 47 us
// (127).
constexpr float SMALL_UNIT = 1024.f;   // (of everything held: coefficients of 60 together keep P in fp16's range)
constexpr int SMALL_THREADS = 512, SMALL_GROUPS = SMALL_THREADS / 128, SMALL_MOST = 256, SMALL_COLUMNS = 256, SMALL_BYTES = 225 * 1024;

struct SmallArgs {
    const void *update[SMALL_MOST], *grad[SMALL_MOST];
    void *out[SMALL_MOST];
    int index[SMALL_MOST], rows[SMALL_MOST], cols[SMALL_MOST];
    float scale[SMALL_MOST];
    float coefficients[DESLOC_MAX_NEWTON_SCHULZ][3];
    int steps;
    float beta, eps, rho, decay;
    int update_bf16, grad_bf16, out_bf16;
    float *const *u_table, *const *x_table;
    int *err;
    int wait_limit;
};

struct SmallPlan {
    int n, m, rows, blocks, square_blocks;   // the sides; rows of a block of 64 columns; such blocks of X and of G
    __host__ __device__ SmallPlan(int r, int c)
        : n(r < c ? r : c), m(r < c ? c : r), rows((n + 15) / 16 * 16), blocks((m + 63) / 64), square_blocks((n + 63) / 64) {}
    __host__ __device__ int half() const { return rows * 128; }                        // bytes of a block
    __host__ __device__ int x_bytes() const { return blocks * half(); }                // hi; lo follows
    __host__ __device__ int g_bytes() const { return square_blocks * half(); }
    // (the products read 128 rows wherever they begin: what lies behind the last ones is never looked at)
    __host__ __device__ int bytes() const { return 2 * x_bytes() + 2 * g_bytes() + (128 - (rows < 128 ? rows : 128)) * 128; }
};

__device__ __forceinline__ int place(const SmallPlan &p, int row, int col) {
    return (col >> 6) * p.half() + row * 128 + ((((col >> 3) & 7) ^ (row & 7)) << 4) + (col & 7) * 2;
}

// Sixteen values of a row as hi and lo; col is a multiple of 16.
__device__ __forceinline__ void put_row(char *hi, int lo, const SmallPlan &p, int row, int col, const float (&v)[16]) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        uint32_t h[4], l[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float a = v[8 * c + 2 * e], b = v[8 * c + 2 * e + 1];
            h[e] = pack_f16(a, b);
            const float2 x = unpack_f16(h[e]);
            l[e] = pack_f16(a - x.x, b - x.y);
        }
        char *const to = hi + place(p, row, col + 8 * c);
        *reinterpret_cast<uint4 *>(to) = make_uint4(h[0], h[1], h[2], h[3]);
        *reinterpret_cast<uint4 *>(to + lo) = make_uint4(l[0], l[1], l[2], l[3]);
    }
}

// Products of `k` (a multiple of 16): A from `a`, k-major, its columns in blocks of `a_block` bytes; B from `b`, k-major like A, or (mn) n-major.  Three of them: hi hi, hi lo, lo hi.
__device__ __forceinline__ void products(uint32_t d, uint32_t a, int a_lo, int a_block, uint32_t b, int b_lo, int b_block, bool mn, int k, uint32_t idesc) {
    const auto desc = [](uint32_t at, int block, bool n_major) {
        return static_cast<uint64_t>((at >> 4) & 0x3fff) | (static_cast<uint64_t>(n_major ? block >> 4 : 1) << 16) | (static_cast<uint64_t>(1024 >> 4) << 32) | (1ull << 46) |
               (2ull << 61);
    };
    for (int which = 0; which < 3; ++which) {
        const uint32_t from_a = a + (which == 2 ? a_lo : 0), from_b = b + (which == 1 ? b_lo : 0);
        for (int x = 0; x < k; x += 16) {
            const uint32_t at_a = from_a + (x >> 6) * a_block + (x & 63) * 2, at_b = mn ? from_b + x * 128 : from_b + (x >> 6) * b_block + (x & 63) * 2;
            mma_f16<1>(d, desc(at_a, 0, false), desc(at_b, b_block, mn), idesc | (mn ? 1u << 16 : 0), which > 0 || x > 0);
        }
    }
}

__global__ void __launch_bounds__(SMALL_THREADS) orth_small_kernel(const __grid_constant__ SmallArgs a) {
    extern __shared__ __align__(1024) char small_smem[];
    __shared__ __align__(8) uint64_t done;
    __shared__ uint32_t tmem_at;
    __shared__ double sums[SMALL_THREADS / 32];
    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0), lane = threadIdx.x & 31, tid = threadIdx.x, which = blockIdx.x;
    const uint32_t pad = (1024 - (smem_u32(small_smem) & 1023)) & 1023;
    const SmallPlan p(a.rows[which], a.cols[which]);
    char *const x = small_smem + pad, *const g = x + 2 * p.x_bytes();
    const int row = 32 * (warp & 3) + lane, group = warp >> 2;   // of the sums: a row per lane, 16 columns at a time
    if (tid == 0) {
        bar_init(&done, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 256;" :: "r"(smem_u32(&tmem_at)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        begin_and_let_next_begin();   // (not before this block has its TMEM: the next kernel's may take all of an SM's and wait for this one's end)
    }
    for (int i = tid * 16; i < 2 * p.x_bytes() + 2 * p.g_bytes(); i += SMALL_THREADS * 16) *reinterpret_cast<uint4 *>(x + i) = make_uint4(0, 0, 0, 0);
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const uint32_t tmem = tmem_at;
    wait_for_earlier_kernels();

    // The norm (squares up to four at a time in fp32, then in fp64), and X.
    const void *const u = a.update[which] ? a.update[which] : a.u_table[a.index[which]];
    const void *const gr = a.grad[which];
    const int cols = a.cols[which], count = a.rows[which] * cols;
    const bool tall = a.rows[which] > cols;
    const float beta = a.beta, rest = 1.f - a.beta, rho = a.rho;
    // Eight times N neighbouring elements a thread, all of them on their way at once; N = 4 where rows allow it.
    constexpr int AHEAD = 8;
    const auto go = [&](auto width) {
        constexpr int N = decltype(width)::value;
        float v[AHEAD][N];
        const auto fetch = [&](int i0) {
#pragma unroll
            for (int e = 0; e < AHEAD; ++e) {
                const int i = i0 + e * SMALL_THREADS * N;
#pragma unroll
                for (int k = 0; k < N; ++k) v[e][k] = 0.f;
                if (i < count) {
                    if (a.update_bf16) load_values(static_cast<const __nv_bfloat16 *>(u) + i, v[e]);
                    else load_values(static_cast<const float *>(u) + i, v[e]);
                }
            }
            if (!gr) return;
#pragma unroll
            for (int e = 0; e < AHEAD; ++e) {
                const int i = i0 + e * SMALL_THREADS * N;
                float w[N] = {};
                if (i < count) {
                    if (a.grad_bf16) load_values(static_cast<const __nv_bfloat16 *>(gr) + i, w);
                    else load_values(static_cast<const float *>(gr) + i, w);
                }
#pragma unroll
                for (int k = 0; k < N; ++k) v[e][k] = beta * v[e][k] + rest * clipped(w[k], rho);
            }
        };
        constexpr int EACH = AHEAD * SMALL_THREADS * N;
        double sum = 0;
        for (int i0 = tid * N; i0 < count; i0 += EACH) {
            fetch(i0);
#pragma unroll
            for (int e = 0; e < AHEAD; ++e) {
                float part = 0;
#pragma unroll
                for (int k = 0; k < N; ++k) part += v[e][k] * v[e][k];
                sum += part;
            }
        }
#pragma unroll
        for (int d = 16; d; d /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        if (lane == 0) sums[warp] = sum;
        __syncthreads();
        sum = 0;
#pragma unroll
        for (int w = 0; w < SMALL_THREADS / 32; ++w) sum += sums[w];
        const float factor = static_cast<float>(static_cast<double>(SMALL_UNIT) / (sqrt(sum) + static_cast<double>(a.eps)));
        const int x_lo = p.x_bytes();
        for (int i0 = tid * N; i0 < count; i0 += EACH) {
            if (count > EACH) fetch(i0);   // (else they are still here)
#pragma unroll
            for (int e = 0; e < AHEAD; ++e) {
                const int i = i0 + e * SMALL_THREADS * N, r = i / cols, c = i - r * cols;
                if (i >= count) break;
                __half h[N], l[N];
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    const float y = v[e][k] * factor;
                    h[k] = __float2half_rn(y);
                    l[k] = __float2half_rn(y - __half2float(h[k]));
                }
                if (N == 4 && !tall) {
                    char *const to = x + place(p, r, c);
                    *reinterpret_cast<uint2 *>(to) = *reinterpret_cast<const uint2 *>(h);
                    *reinterpret_cast<uint2 *>(to + x_lo) = *reinterpret_cast<const uint2 *>(l);
                } else {
#pragma unroll
                    for (int k = 0; k < N; ++k) {
                        char *const to = x + (tall ? place(p, c + k, r) : place(p, r, c + k));
                        *reinterpret_cast<__half *>(to) = h[k];
                        *reinterpret_cast<__half *>(to + x_lo) = l[k];
                    }
                }
            }
        }
    };
    const uintptr_t low = (reinterpret_cast<uintptr_t>(u) & (a.update_bf16 ? 7u : 15u)) | (reinterpret_cast<uintptr_t>(gr) & (a.grad_bf16 ? 7u : 15u));
    if (cols % 4 == 0 && low == 0) go(std::integral_constant<int, 4>());
    else go(std::integral_constant<int, 1>());

    const uint32_t at_x = smem_u32(x), at_g = smem_u32(g);
    const uint32_t idesc = 1u << 4 | static_cast<uint32_t>(GEMM_BM >> 4) << 24;
    const auto of_n = [](int n) { return static_cast<uint32_t>(n >> 3) << 17; };
    uint32_t phase = 0;
    bool ok = true;
    // Everybody's writes are operands from here on; the products; everybody may look at the sums.
    const auto run = [&](const auto &issue) {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        tmem_fence_before();
        __syncthreads();
        if (warp == 0 && elect_one()) {
            tmem_fence_after();
            issue();
            mma_commit<1>(&done);
        }
        __syncwarp();
        const bool came = bar_wait(&done, phase, a.wait_limit);
        if (__syncthreads_or(!came)) {
            if (tid == 0 && a.err) *reinterpret_cast<volatile int *>(a.err) = 1;
            bar_wait(&done, phase, GEMM_DRAIN_LIMIT);
            return false;
        }
        phase ^= 1;
        tmem_fence_after();
        return true;
    };
    for (int step = 0; step < a.steps && ok; ++step) {
        const float ca = a.coefficients[step][0] * SMALL_UNIT, cb = a.coefficients[step][1], cc = a.coefficients[step][2] / SMALL_UNIT;
        const uint32_t lanes = static_cast<uint32_t>(32 * (warp & 3)) << 16;
        ok = run([&] { products(tmem, at_x, p.x_bytes(), p.half(), at_x, p.x_bytes(), p.half(), false, (p.m + 15) / 16 * 16, idesc | of_n(p.rows)); });
        if (!ok) break;
        for (int c = 16 * group; c < p.rows; c += 16 * SMALL_GROUPS) {
            float v[16];
            tmem_load16(tmem + lanes + c, v);
            tmem_wait();
            if (row < p.rows) {
#pragma unroll
                for (int e = 0; e < 16; ++e) v[e] *= 1.f / SMALL_UNIT;
                put_row(g, p.g_bytes(), p, row, c, v);
            }
        }
        ok = run([&] { products(tmem, at_g, p.g_bytes(), p.half(), at_g, p.g_bytes(), p.half(), false, p.rows, idesc | of_n(p.rows)); });
        if (!ok) break;
        for (int c = 16 * group; c < p.rows; c += 16 * SMALL_GROUPS) {
            float v[16];
            tmem_load16(tmem + lanes + c, v);
            tmem_wait();
            if (row < p.rows) {
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const char *const from = g + place(p, row, c + 8 * half);
                    const uint4 h = *reinterpret_cast<const uint4 *>(from), l = *reinterpret_cast<const uint4 *>(from + p.g_bytes());
                    const uint32_t hw[4] = {h.x, h.y, h.z, h.w}, lw[4] = {l.x, l.y, l.z, l.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float2 hh = unpack_f16(hw[e]), ll = unpack_f16(lw[e]);
                        const int k = 8 * half + 2 * e;
                        v[k] = cc * v[k] + cb * (hh.x + ll.x) + (c + k == row ? ca : 0.f);
                        v[k + 1] = cc * v[k + 1] + cb * (hh.y + ll.y) + (c + k + 1 == row ? ca : 0.f);
                    }
                }
                put_row(g, p.g_bytes(), p, row, c, v);   // (each lane where it has read; nobody reads G again)
            }
        }
        const bool last = step + 1 == a.steps;
        for (int c0 = 0; c0 < p.m && ok; c0 += SMALL_COLUMNS) {
            const int some = min(SMALL_COLUMNS, (p.m - c0 + 15) / 16 * 16);
            const uint32_t from = at_x + (c0 >> 6) * p.half();
            ok = run([&] { products(tmem, at_g, p.g_bytes(), p.half(), from, p.x_bytes(), p.half(), true, p.rows, idesc | of_n(some)); });
            if (!ok) break;
            for (int c = 16 * group; c < some; c += 16 * SMALL_GROUPS) {
                float v[16];
                tmem_load16(tmem + lanes + c, v);
                tmem_wait();
                if (!last) {
                    if (row < p.rows) {
#pragma unroll
                        for (int e = 0; e < 16; ++e) v[e] *= 1.f / SMALL_UNIT;
                        put_row(x, p.x_bytes(), p, row, c0 + c, v);   // (columns that no other part of X comes from)
                    }
                } else if (row < p.n) {
                    const float scale = a.scale[which] / (SMALL_UNIT * SMALL_UNIT);
                    const bool step_of_x = !a.out[which];
                    float *const to = static_cast<float *>(step_of_x ? a.x_table[a.index[which]] : a.out[which]);
                    const int col0 = c0 + c, each = tall ? cols : 1, left = p.m - col0;
                    const int i = tall ? col0 * cols + row : row * cols + col0;
                    float was[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) was[e] = step_of_x && e < left ? to[i + e * each] : 0.f;
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        v[e] = step_of_x ? a.decay * was[e] - scale * v[e] : scale * v[e];
                        if (e >= left) continue;
                        if (a.out_bf16) reinterpret_cast<__nv_bfloat16 *>(to)[i + e * each] = __float2bfloat16_rn(v[e]);
                        else to[i + e * each] = v[e];
                    }
                }
            }
        }
    }
    tmem_fence_before();
    __syncthreads();
    if (warp == 1) {
        tmem_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 256;" :: "r"(tmem) : "memory");
    }
}

}  // namespace

bool orth_is_small(int rows, int cols) {
    const int64_t n = std::min(rows, cols), m = std::max(rows, cols);
    return n <= 128 && m <= 4096 && SmallPlan(rows, cols).bytes() + 1024 <= SMALL_BYTES;
}

cudaError_t launch_orth_small(const OrthArgs &a, int first, int count, int *err, int wait_limit, cudaStream_t stream, int *launches) {
    static thread_local SmallArgs s;
    static std::atomic<uint64_t> ready{0};
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e == cudaSuccess && (device >= 64 || !(ready.load() >> device & 1))) {
        e = cudaFuncSetAttribute(orth_small_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SMALL_BYTES);
        if (e == cudaSuccess && device < 64) ready.fetch_or(1ull << device);
    }
    for (int at = first; e == cudaSuccess && at < first + count; at += SMALL_MOST) {
        const int some = std::min(SMALL_MOST, first + count - at);
        int bytes = 0;
        for (int i = 0; i < some; ++i) {
            const OrthMatrix &m = a.list[at + i];
            s.update[i] = m.update, s.grad[i] = m.grad, s.out[i] = m.out, s.index[i] = m.index, s.rows[i] = m.rows, s.cols[i] = m.cols, s.scale[i] = m.scale;
            bytes = std::max(bytes, SmallPlan(m.rows, m.cols).bytes());
        }
        std::memcpy(s.coefficients, a.coefficients, sizeof(float) * 3 * a.steps);
        s.steps = a.steps, s.beta = a.beta, s.eps = a.eps, s.rho = a.rho, s.decay = a.decay;
        s.update_bf16 = a.update_bf16, s.grad_bf16 = a.grad_bf16, s.out_bf16 = a.out_bf16;
        s.u_table = a.u_table, s.x_table = a.x_table, s.err = err, s.wait_limit = wait_limit;
        cudaLaunchConfig_t lc{};
        lc.gridDim = dim3(static_cast<unsigned>(some));
        lc.blockDim = dim3(SMALL_THREADS);
        lc.dynamicSmemBytes = static_cast<size_t>(bytes) + 1024;
        lc.stream = stream;
        cudaLaunchAttribute overlap{};
        overlap.id = cudaLaunchAttributeProgrammaticStreamSerialization;
        overlap.val.programmaticStreamSerializationAllowed = 1;
        lc.attrs = &overlap;
        lc.numAttrs = 1;
        void *args[1] = {&s};
        e = cudaLaunchKernelExC(&lc, reinterpret_cast<const void *>(orth_small_kernel), args);
        if (e == cudaSuccess) ++*launches;
    }
    return e;
}

}  // namespace desloc
