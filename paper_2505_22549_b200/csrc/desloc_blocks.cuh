// Launchers of the gated feed-forward block and of the orthogonalised updates.
#pragma once
#include "desloc_ops.cuh"

namespace desloc {

// The block's sizes and operands; per worker m: h at h + m * hs0, weights at gate[m], up[m] [hidden, width], down[m] [width, hidden].  All bf16.
struct FfnArgs {
    int M, tokens, width, hidden;
    const void *h;
    long long hs0, hs1;
    const void *gate[DESLOC_MAX_M], *up[DESLOC_MAX_M], *down[DESLOC_MAX_M];
    // forward
    void *y;
    long long ys0, ys1;
    void *kept_gate, *kept_up;   // [M][tokens][hidden], or null
    // backward
    const void *was_gate, *was_up;
    const void *dy;
    long long dys0, dys1;
    void *dh;
    long long dhs0, dhs1;
    void *dgate[DESLOC_MAX_M], *dup[DESLOC_MAX_M], *ddown[DESLOC_MAX_M];
    int accumulate, grad_bf16;
};
// Bytes of working memory.
int64_t ffn_work(const FfnArgs &a, bool backward);
cudaError_t launch_ffn(const FfnArgs &a, char *work, int *err, int wait_limit, cudaStream_t stream, int *launches);
cudaError_t launch_ffn_grad(const FfnArgs &a, char *work, int *err, int wait_limit, cudaStream_t stream, int *launches);

// A list of matrices, any order: number `index` in the context's tables, or addresses.
struct OrthMatrix {
    int rows, cols, index;
    const void *update, *grad;   // update: null where the tables say
    void *out;                   // null: a step of x
    float scale;                 // of the result, with the learning rate; filled in by launch_orth()
};
struct OrthArgs {
    OrthMatrix *list;            // sorted in place
    int count, steps;
    const float *coefficients;   // [steps][3]
    float eps, beta, rho;        // of the look-ahead beta * update + (1 - beta) * grad, grad clipped to +-rho (infinity: not at all)
    bool update_bf16, grad_bf16, out_bf16;
    float *const *u_table, *const *x_table;   // on the device
    int scale;                   // desloc_scale_t
    float lr, decay;             // of the step: x := decay * x - lr * scale * result
};
// A gradient as the step has it in the momentum: sgn(g) min(|g|, rho).  (NaN stays NaN, so that the result shows it.)
__device__ __forceinline__ float clipped(float g, float rho) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;\n min.NaN.f32 %0, %0, %3;" : "=&f"(r) : "f"(g), "f"(-rho), "f"(rho));
    return r;
}
// Whether a matrix is taken by a block of its own, and the launch of such ones: list[first, first + count).
bool orth_is_small(int rows, int cols);
cudaError_t launch_orth_small(const OrthArgs &a, int first, int count, int *err, int wait_limit, cudaStream_t stream, int *launches);
int64_t orth_work(const OrthArgs &a);
cudaError_t launch_orth(const OrthArgs &a, char *work, int *err, int wait_limit, cudaStream_t stream, int *launches);

}  // namespace desloc
