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

#include "linear_kernels.cuh"

namespace e3j {
namespace layer {
namespace {

// Status word of these kernels (0 = fine, 1 = a bounded wait gave up and the output is invalid): read and cleared by
// e3j_linear_status.
__device__ int32_t g_linear_status;

constexpr int kMostWidth = 4096;
constexpr size_t kSmemOfSm = 227 * 1024, kSmemOfBlock = 227 * 1024;

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

template <Product P, class T, class G, int NT>
struct Launch {
    using L = LinTile<P, T, G, NT>;
    // stages, resident chunks of B and blocks an SM for `chunks` chunks
    static int shape(LinArgs& a, int chunks, size_t& smem) {
        for (int blocks = L::kBlocks; blocks >= 1; --blocks) {
            const size_t fixed = 1024 + (P == kGradW ? 16 * NT * sizeof(float) : NT * sizeof(float)) + 256;
            const size_t room = std::min(kSmemOfSm / blocks, kSmemOfBlock + 1024) - fixed;
            for (int resident = P == kGradW ? 0 : 1; resident >= 0; --resident)
                for (int stages = 2; stages >= 1; --stages) {
                    smem = L::smem_bytes(stages, resident ? chunks : stages);
                    if (smem > room) continue;
                    a.stages = stages;
                    a.resident = resident;
                    return blocks;
                }
        }
        return 0;
    }
    static int run(LinArgs& a, cudaStream_t st) {
        static std::atomic<uint64_t> allowed{0};   // bit per device
        int dev = 0;
        E3J_CUDA_TRY(cudaGetDevice(&dev));
        if (dev < 0 || dev >= 64) return E3J_ERR_UNSUPPORTED;
        if (!(allowed.load(std::memory_order_relaxed) >> dev & 1)) {
            const size_t statics = P == kGradW ? 16 * NT * sizeof(float) + 256 : NT * sizeof(float) + 256;
            E3J_CUDA_TRY(cudaFuncSetAttribute(linear_kernel<P, T, G, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                              (int)(kSmemOfBlock - statics)));
            allowed.fetch_or(1ull << dev, std::memory_order_relaxed);
        }
        if (int rc = status_word(&a.status)) return rc;
        const int columns = P == kGradX ? a.n_in : a.n_out;
        a.n_tiles = (columns + NT - 1) / NT;
        size_t smem = 0;
        const int blocks = shape(a, P == kGradW ? kGroupChunks : ((P == kGradX ? a.n_out : a.n_in) + kChunk - 1) / kChunk, smem);
        if (blocks == 0) return E3J_ERR_UNSUPPORTED;
        int64_t grid;
        if (P == kGradW) {
            grid = (int64_t)a.n_tiles * a.m_tiles * a.ranges;
        } else {
            const int64_t row_tiles = (a.rows + kTileRows - 1) / kTileRows;
            const int64_t per = std::max<int64_t>((int64_t)sm_count() * blocks / a.n_tiles, 1);
            grid = a.n_tiles * std::min(per, row_tiles);
        }
        return launch_dependent(linear_kernel<P, T, G, NT>, dim3((unsigned)grid), dim3(kLinThreads), smem, st, a);
    }
};

template <Product P, class T, class G> int product(LinArgs& a, cudaStream_t st) {
    return (P == kGradX ? a.n_in : a.n_out) <= 64 ? Launch<P, T, G, 64>::run(a, st) : Launch<P, T, G, 128>::run(a, st);
}

inline bool whole(const void* p, int64_t ld, size_t size, size_t bytes) { return (((uintptr_t)p | (uintptr_t)(ld * size)) & (bytes - 1)) == 0; }

// ---- backward: [gz | shares]
struct BwdLayout { int64_t ld_gz; int n_tiles, m_tiles, ranges; size_t gz, shares, total; };
BwdLayout bwd_layout(int64_t rows, int n_in, int n_out, int act) {
    BwdLayout L{};
    L.ld_gz = align_up(n_out, 8);
    const int nt = n_out <= 64 ? 64 : 128;
    L.n_tiles = (n_out + nt - 1) / nt;
    L.m_tiles = (n_in + kTileRows - 1) / kTileRows;
    const int64_t chunks = std::max<int64_t>((rows + kChunk - 1) / kChunk, 1);
    const int64_t resident = (int64_t)sm_count() * (nt == 64 ? 2 : 1);
    L.ranges = (int)std::min(std::max<int64_t>(resident / (L.n_tiles * L.m_tiles), 1), chunks);
    L.shares = act == E3J_ACT_NONE ? 0 : align_up((size_t)rows * L.ld_gz * sizeof(float), 256);
    L.total = L.shares + align_up((size_t)L.ranges * ((size_t)n_in * n_out + n_out) * sizeof(float), 256);
    return L;
}

int linear_args_status(int dtype, int64_t rows, int n_in, int n_out, int act) {
    if (rows < 0 || n_in < 1 || n_out < 1 || dtype < E3J_F32 || dtype > E3J_BF16 || act < E3J_ACT_NONE || act > E3J_ACT_GELU)
        return E3J_ERR_INVALID_ARG;
    return n_in > kMostWidth || n_out > kMostWidth || rows >= (1ll << 31) - 1 ? E3J_ERR_UNSUPPORTED : E3J_OK;
}

template <class T> int linear_fwd(LinArgs& a, cudaStream_t st) {
    a.vector = (whole(a.x, a.n_in, sizeof(T), 16) ? 1u : 0u) | (whole(a.W, a.n_out, sizeof(T), 16) ? 2u : 0u) |
               (whole(a.out, a.n_out, sizeof(T), 4 * sizeof(T)) ? 4u : 0u) | (whole(a.residual, a.n_out, sizeof(T), 4 * sizeof(T)) ? 8u : 0u);
    return product<kForward, T, T>(a, st);
}

template <class T, class G> int gradients(LinArgs a, const BwdLayout& L, void* grad_x, void* grad_W, void* grad_b, cudaStream_t st) {
    const unsigned x16 = whole(a.x, a.n_in, sizeof(T), 16), W16 = whole(a.W, a.n_out, sizeof(T), 16), gz16 = whole(a.gz, a.ld_gz, sizeof(G), 16);
    if (grad_x) {
        a.out = grad_x;
        a.vector = gz16 | W16 << 1 | (whole(grad_x, a.n_in, sizeof(T), 4 * sizeof(T)) ? 4u : 0u);
        if (int rc = product<kGradX, T, G>(a, st)) return rc;
    }
    if (!grad_W && !grad_b) return E3J_OK;
    a.vector = x16 | gz16 << 1;
    a.ranges = L.ranges;
    a.m_tiles = L.m_tiles;
    a.want_sums = grad_b != nullptr;
    if (int rc = product<kGradW, T, G>(a, st)) return rc;
    return sum_shares<T>(L.ranges, (int64_t)a.n_in * a.n_out, a.n_out, a.shares, (T*)grad_W, (T*)grad_b, st);
}

template <class T>
int linear_bwd(LinArgs& a, const BwdLayout& L, void* workspace, void* grad_x, void* grad_W, void* grad_b, cudaStream_t st) {
    a.shares = (float*)((char*)workspace + L.shares);
    if (a.act == E3J_ACT_NONE) {
        a.gz = a.grad_y;
        a.ld_gz = a.n_out;
        return gradients<T, T>(a, L, grad_x, grad_W, grad_b, st);
    }
    a.out = workspace;
    a.ld_gz = (int)L.ld_gz;
    a.vector = (whole(a.x, a.n_in, sizeof(T), 16) ? 1u : 0u) | (whole(a.W, a.n_out, sizeof(T), 16) ? 2u : 0u) |
               (whole(a.grad_y, a.n_out, sizeof(T), 4 * sizeof(T)) ? 8u : 0u);
    if (int rc = product<kSlope, T, float>(a, st)) return rc;
    a.gz = workspace;
    return gradients<T, float>(a, L, grad_x, grad_W, grad_b, st);
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
    LinArgs a{};
    a.rows = rows; a.n_in = n_in; a.n_out = n_out; a.act = act; a.n_real = n_real;
    a.x = x; a.W = W; a.b = b; a.residual = residual; a.out = y;
    return dtype == E3J_F32 ? linear_fwd<float>(a, (cudaStream_t)stream) : linear_fwd<bf16>(a, (cudaStream_t)stream);
}

size_t e3j_linear_bwd_workspace_bytes(int dtype, int64_t rows, int n_in, int n_out, int act) {
    if (linear_args_status(dtype, rows, n_in, n_out, act) != E3J_OK) return 0;
    return bwd_layout(rows, n_in, n_out, act).total;
}

int e3j_linear_bwd(int dtype, int64_t rows, int n_in, int n_out, const void* x, const void* W, const void* b, const void* grad_y,
                   int act, const int32_t* n_real, void* grad_x, void* grad_W, void* grad_b, void* workspace,
                   size_t workspace_bytes, void* stream) {
    if (int rc = linear_args_status(dtype, rows, n_in, n_out, act)) return rc;
    cudaStream_t st = (cudaStream_t)stream;
    const size_t size = dtype == E3J_F32 ? 4 : 2;
    const uintptr_t arrays = (uintptr_t)x | (uintptr_t)W | (uintptr_t)b | (uintptr_t)grad_y | (uintptr_t)grad_x |
                             (uintptr_t)grad_W | (uintptr_t)grad_b;
    if (arrays & (size - 1)) return E3J_ERR_INVALID_ARG;
    if (rows == 0) {   // sums over no rows
        if (grad_W) E3J_CUDA_TRY(cudaMemsetAsync(grad_W, 0, size * n_in * n_out, st));
        if (grad_b) E3J_CUDA_TRY(cudaMemsetAsync(grad_b, 0, size * n_out, st));
        return E3J_OK;
    }
    if (!x || !W || !grad_y) return E3J_ERR_INVALID_ARG;
    if (!grad_x && !grad_W && !grad_b) return E3J_OK;
    const BwdLayout L = bwd_layout(rows, n_in, n_out, act);
    if (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < L.total) return E3J_ERR_WORKSPACE;
    LinArgs a{};
    a.rows = rows; a.n_in = n_in; a.n_out = n_out; a.act = act; a.n_real = n_real;
    a.x = x; a.W = W; a.b = b; a.grad_y = grad_y;
    return dtype == E3J_F32 ? linear_bwd<float>(a, L, workspace, grad_x, grad_W, grad_b, st)
                            : linear_bwd<bf16>(a, L, workspace, grad_x, grad_W, grad_b, st);
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
