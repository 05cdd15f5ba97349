// Linear layer with bias, activation and residual, forward and backward: the radial network's hidden layers, on edges, and the
// read-out or mixing of node scalars.
//
//   y = act(x W + b) + residual
//   backward, from x, W, b and g = grad_y:  gz = g act'(x W + b);  grad_x = gz W^T;  grad_W = x^T gz;  grad_b = sum_rows gz
//   (grad_residual = g)
//
// The backward forms x W + b again instead of having the forward keep it: the layer saves nothing but its own input.  Without
// an activation gz is g.  The kernels are in linear_kernels.cuh.
#include <algorithm>
#include <atomic>

#include "layer_common.cuh"
#include "linear.hpp"

namespace e3j {
namespace layer {
namespace {

// Status word of these kernels (0 = fine, 1 = a bounded wait gave up and the output is invalid): read and cleared by
// e3j_linear_status.
__device__ int32_t g_linear_status;

constexpr int kMostWidth = 4096;

int status_word(int32_t** word) {
    static std::atomic<int32_t*> of_device[64];
    int dev = 0;
    E3J_CUDA_TRY(cudaGetDevice(&dev));
    if (dev < 0 || dev >= 64) return E3J_ERR_UNSUPPORTED;
    int32_t* w = of_device[dev].load(std::memory_order_acquire);
    if (!w) {
        void* p = nullptr;
        E3J_CUDA_TRY(cudaGetSymbolAddress(&p, g_linear_status));
        of_device[dev].store(w = (int32_t*)p, std::memory_order_release);
    }
    *word = w;
    return E3J_OK;
}

BwdLayout bwd_layout(int dtype, int64_t rows, int n_in, int n_out, int act) {
    BwdLayout L{};
    const size_t share = ((size_t)n_in * n_out + n_out) * sizeof(float);
    L.narrow = n_in <= 64 && n_out <= 64;
    if (L.narrow) {
        L.ranges = (int)std::min<int64_t>(std::max<int64_t>((rows + 127) / 128, 1), sm_count());
        L.direct = L.ranges <= kClusterBlocks;   // (1201 rows as two tiles a block: 14.7 us; ten blocks and a kernel for the sums: 13)
        L.total = L.direct ? 0 : align_up(L.ranges * (dtype == E3J_F32 ? 2 : 1) * share, 256);   // (float32: two shares a block)
        return L;
    }
    L.ld_gz = align_up(n_out, 8);
    const int nt = n_out <= 64 ? 64 : 128;
    const int n_tiles = (n_out + nt - 1) / nt;
    L.m_tiles = (n_in + 127) / 128;
    const int64_t chunks = std::max<int64_t>((rows + 63) / 64, 1);
    L.ranges = chunks <= 4 ? 1 : (int)std::min(std::max<int64_t>(sm_count() / (n_tiles * L.m_tiles), 1), chunks);
    L.direct = L.ranges == 1;
    L.shares = act == E3J_ACT_NONE ? 0 : align_up((size_t)rows * L.ld_gz * sizeof(float), 256);
    L.total = L.shares + (L.direct ? 0 : align_up(L.ranges * share, 256));
    return L;
}

int linear_args_status(int dtype, int64_t rows, int n_in, int n_out, int act) {
    if (rows < 0 || n_in < 1 || n_out < 1 || dtype < E3J_F32 || dtype > E3J_BF16 || act < E3J_ACT_NONE || act > E3J_ACT_GELU)
        return E3J_ERR_INVALID_ARG;
    return n_in > kMostWidth || n_out > kMostWidth || rows >= (1ll << 31) - 1 ? E3J_ERR_UNSUPPORTED : E3J_OK;
}

}  // namespace
}  // namespace layer
}  // namespace e3j

using namespace e3j;
using namespace e3j::layer;

extern "C" {

int e3j_linear_fwd(int dtype, int64_t rows, int n_in, int n_out, const void* x, const void* W, const void* b, const void* residual,
                   int act, const int32_t* n_real, void* y, void* stream) {
    if (int rc = linear_args_status(dtype, rows, n_in, n_out, act)) return rc;
    if (rows == 0) return E3J_OK;
    if (!x || !W || !y) return E3J_ERR_INVALID_ARG;
    const uintptr_t odd = dtype == E3J_F32 ? 3u : 1u;
    if (((uintptr_t)x | (uintptr_t)W | (uintptr_t)b | (uintptr_t)residual | (uintptr_t)y) & odd) return E3J_ERR_INVALID_ARG;
    if ((uintptr_t)n_real & 3u) return E3J_ERR_INVALID_ARG;
    LinArgs a{};
    a.rows = rows; a.n_in = n_in; a.n_out = n_out; a.n_real = n_real;
    if (int rc = status_word(&a.status)) return rc;
    a.x = x; a.W = W; a.b = b; a.residual = residual; a.out = y;
    return dtype == E3J_F32 ? linear_fwd<float>(a, act, (cudaStream_t)stream) : linear_fwd<bf16>(a, act, (cudaStream_t)stream);
}

size_t e3j_linear_bwd_workspace_bytes(int dtype, int64_t rows, int n_in, int n_out, int act) {
    if (linear_args_status(dtype, rows, n_in, n_out, act) != E3J_OK) return 0;
    return bwd_layout(dtype, rows, n_in, n_out, act).total;
}

int e3j_linear_bwd(int dtype, int64_t rows, int n_in, int n_out, const void* x, const void* W, const void* b, const void* grad_y,
                   int act, const int32_t* n_real, void* grad_x, void* grad_W, void* grad_b, void* workspace,
                   size_t workspace_bytes, void* stream) {
    if (int rc = linear_args_status(dtype, rows, n_in, n_out, act)) return rc;
    cudaStream_t st = (cudaStream_t)stream;
    const size_t size = dtype == E3J_F32 ? 4 : 2;
    const uintptr_t arrays = (uintptr_t)x | (uintptr_t)W | (uintptr_t)b | (uintptr_t)grad_y | (uintptr_t)grad_x |
                             (uintptr_t)grad_W | (uintptr_t)grad_b;
    if ((arrays & (size - 1)) || ((uintptr_t)n_real & 3u)) return E3J_ERR_INVALID_ARG;
    if (rows == 0) {   // sums over no rows
        if (grad_W) E3J_CUDA_TRY(cudaMemsetAsync(grad_W, 0, size * n_in * n_out, st));
        if (grad_b) E3J_CUDA_TRY(cudaMemsetAsync(grad_b, 0, size * n_out, st));
        return E3J_OK;
    }
    if (!x || !W || !grad_y) return E3J_ERR_INVALID_ARG;
    if (!grad_x && !grad_W && !grad_b) return E3J_OK;
    const BwdLayout L = bwd_layout(dtype, rows, n_in, n_out, act);
    const size_t need = grad_W || grad_b ? L.total : L.shares;   // (grad_x alone: gz, if that is in memory)
    if (need > 0 && (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < need)) return E3J_ERR_WORKSPACE;
    LinArgs a{};
    a.rows = rows; a.n_in = n_in; a.n_out = n_out; a.n_real = n_real;
    if (int rc = status_word(&a.status)) return rc;
    a.x = x; a.W = W; a.b = b; a.grad_y = grad_y;
    return dtype == E3J_F32 ? linear_bwd<float>(a, act, L, workspace, grad_x, grad_W, grad_b, st)
                            : linear_bwd<bf16>(a, act, L, workspace, grad_x, grad_W, grad_b, st);
}

int e3j_linear_status(int32_t* status) {
    if (!status) return E3J_ERR_INVALID_ARG;
    int32_t* word = nullptr;
    if (int rc = status_word(&word)) return rc;
    E3J_CUDA_TRY(cudaDeviceSynchronize());
    E3J_CUDA_TRY(cudaMemcpy(status, word, sizeof(int32_t), cudaMemcpyDeviceToHost));
    if (*status != 0) E3J_CUDA_TRY(cudaMemset(word, 0, sizeof(int32_t)));
    return E3J_OK;
}

}  // extern "C"
