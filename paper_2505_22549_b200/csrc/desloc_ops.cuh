// Operators around the step: launchers, and what their kernels share.
#pragma once
#include <cmath>

#include <cuda_bf16.h>

#include "../../include/desloc.h"
#include "desloc_kernels.cuh"

namespace desloc {

// Token numbers: element (m, i) at m * s0 + i * s1.
struct TokenRows {
    const void *data;
    long long s0, s1;
    int wide;   // 64-bit numbers
};

// What the entry points ask of rows that they are given: a known type, and data on a boundary of it.
inline bool is_value_rows(const desloc_rows &r) {
    return (r.dtype == DESLOC_F32 || r.dtype == DESLOC_BF16) && reinterpret_cast<uintptr_t>(r.data) % (r.dtype == DESLOC_F32 ? 4 : 2) == 0;
}
inline bool is_token_rows(const desloc_rows &r) {
    return (r.dtype == DESLOC_I32 || r.dtype == DESLOC_I64) && reinterpret_cast<uintptr_t>(r.data) % (r.dtype == DESLOC_I64 ? 8 : 4) == 0;
}
// Whether rows of `width` elements that are written share some: of the two strides the smaller one (over what it reaches) has to pass a row, the larger
// one all of those.  (In double: strides and counts are the caller's, and a product may leave 64 bits.)
inline bool rows_overlap(const desloc_rows &r, int64_t outer, int64_t inner, int64_t width) {
    double s[2] = {std::fabs(static_cast<double>(r.stride[0])), std::fabs(static_cast<double>(r.stride[1]))};
    double n[2] = {static_cast<double>(outer), static_cast<double>(inner)};
    const int first = n[1] <= 1 || (n[0] > 1 && s[0] < s[1]) ? 0 : 1;
    const double reach = n[first] <= 1 ? width : s[first] * (n[first] - 1) + width;
    return (n[first] > 1 && s[first] < width) || (n[1 - first] > 1 && s[1 - first] < reach);
}
inline TokenRows token_rows(const desloc_rows &r) { return {r.data, r.stride[0], r.stride[1], r.dtype == DESLOC_I64}; }

// Number of the token at element `at`; -1 where it is outside [0, vocab), which is compared in 64 bits.
__device__ __forceinline__ int token_at(const TokenRows &t, long long at, int vocab) {
    const long long v = t.wide ? static_cast<const long long *>(t.data)[at] : static_cast<const int *>(t.data)[at];
    return v >= 0 && v < vocab ? static_cast<int>(v) : -1;
}

// N consecutive values as fp32, aligned to min(N * sizeof(T), 16) bytes; N = 1, 2, 4 or 8.
template <int N, typename T>
__device__ __forceinline__ void load_values(const T *p, float (&f)[N]) {
    if constexpr (N == 1) {
        f[0] = static_cast<float>(*p);
    } else if constexpr (N == 2 && sizeof(T) == 4) {
        const float2 v = *reinterpret_cast<const float2 *>(p);
        f[0] = v.x, f[1] = v.y;
    } else if constexpr (N == 2) {
        const uint32_t w = *reinterpret_cast<const uint32_t *>(p);
        f[0] = __uint_as_float(w << 16), f[1] = __uint_as_float(w & 0xffff0000u);
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int k = 0; k < N; k += 4) {
            const float4 v = *reinterpret_cast<const float4 *>(p + k);
            f[k] = v.x, f[k + 1] = v.y, f[k + 2] = v.z, f[k + 3] = v.w;
        }
    } else {
        uint32_t w[N / 2];
        if constexpr (N == 4) {
            const uint2 v = *reinterpret_cast<const uint2 *>(p);
            w[0] = v.x, w[1] = v.y;
        } else {
            const uint4 v = *reinterpret_cast<const uint4 *>(p);
            w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
        }
#pragma unroll
        for (int k = 0; k < N / 2; ++k) f[2 * k] = __uint_as_float(w[k] << 16), f[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
    }
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}

// The same for stores, rounded to the nearest.
template <int N, typename T>
__device__ __forceinline__ void store_values(T *p, const float (&f)[N]) {
    if constexpr (sizeof(T) == 4) {
        if constexpr (N == 1) {
            *p = f[0];
        } else if constexpr (N == 2) {
            *reinterpret_cast<float2 *>(p) = make_float2(f[0], f[1]);
        } else {
#pragma unroll
            for (int k = 0; k < N; k += 4) *reinterpret_cast<float4 *>(p + k) = make_float4(f[k], f[k + 1], f[k + 2], f[k + 3]);
        }
    } else {
        if constexpr (N == 1) *p = __float2bfloat16_rn(f[0]);
        else if constexpr (N == 2) *reinterpret_cast<uint32_t *>(p) = pack_bf16(f[0], f[1]);
        else if constexpr (N == 4) *reinterpret_cast<uint2 *>(p) = make_uint2(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]));
        else *reinterpret_cast<uint4 *>(p) = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
    }
}

// A launch that may begin while the kernel in front of it still runs (the kernels wait before they touch anything), or, where
// `overlap` is false, one behind it.
template <typename... P, typename... A>
cudaError_t launch_op(void (*kernel)(P...), dim3 grid, dim3 threads, size_t smem, bool overlap, cudaStream_t stream, A... args) {
    cudaLaunchConfig_t lc{};
    lc.gridDim = grid;
    lc.blockDim = threads;
    lc.dynamicSmemBytes = smem;
    lc.stream = stream;
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = &at;
    lc.numAttrs = overlap ? 1 : 0;
    return cudaLaunchKernelEx(&lc, kernel, static_cast<P>(args)...);
}

struct EmbedArgs {
    const float *const *x;   // worker m's table: x[m * x_stride]
    int x_stride;
    TokenRows tokens;
    void *out;
    long long os0, os1;
    int n, vocab, width;
    float scale;
};
cudaError_t launch_embed(const EmbedArgs &a, int M, bool bf16, cudaStream_t stream);

struct EmbedGradArgs {
    TokenRows tokens;
    const void *dout;
    long long ds0, ds1;
    int n, vocab, width;
    float scale;
    int accumulate;
    // How the sort is cut: tokens with the same last `bits` bits go to the same block, which tells `keys` numbers apart.
    int bits, keys;
    int piece, pieces;       // places in a piece of a long run (a power of two), pieces of a worker at most
    int columns;             // groups of columns that a piece's blocks take
    // Working memory, all of it written before it is read.
    unsigned char *seen;     // [M][vocab] whether the token occurs
    int4 *places;            // [M][n] position, token, first place and length of the token's run: sorted by token (the vocabulary in another
                             // order), then by position
    int *count;              // [M] how many of them
    int *tickets;            // [M][pieces][columns]: pieces of a long run that are done, at its first piece
    float *partial;          // [M][pieces][row]: sums of the pieces of long runs
    long long row;
    void *g[DESLOC_MAX_M];
};
// Fills in the plan and the pointers into `work`; the bytes that it takes.
int64_t plan_embed_grad(EmbedGradArgs &a, int M, char *work);
cudaError_t launch_embed_grad(EmbedGradArgs a, int M, bool dout_bf16, bool grad_bf16, cudaStream_t stream, int *launches);

struct LogprobArgs {
    const void *x;
    long long xs0, xs1;
    TokenRows tokens;
    unsigned rows, inner;
    int vocab, top;
    float *logp, *lse, *entropy;
    long long *top_ids;
    float *top_logp;
};
cudaError_t launch_logprobs(const LogprobArgs &a, bool bf16, cudaStream_t stream);

struct LogprobGradArgs {
    const void *x;
    long long xs0, xs1;
    TokenRows tokens;
    unsigned rows, inner;
    int vocab;
    const float *lse, *dlogp, *entropy, *dentropy;
    void *out;
    long long os0, os1;
};
cudaError_t launch_logprobs_grad(const LogprobGradArgs &a, bool bf16, cudaStream_t stream);

}  // namespace desloc
