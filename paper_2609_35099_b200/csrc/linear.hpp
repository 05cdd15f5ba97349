// Between the linear layer's C entry points (linear.cu) and its launches (linear_f32.cu, linear_bf16.cu).
#pragma once
#include <cuda.h>   // CUtensorMap
#include <cuda_runtime.h>

#include <cstddef>
#include <cstdint>

namespace e3j {
namespace layer {

enum Product { kForward, kSlope, kGradX, kGradW };
// kForward  y = act(x W + b) + residual
// kSlope    gz = grad_y act'(x W + b), float32, into the workspace
// kGradX    grad_x = gz W^T
// kGradW    shares of x^T gz and of the column sums of gz, one a range of rows

struct LinArgs {
    CUtensorMap map_a;     // boxes of 128 rows x 64 columns of A, where `boxes` is set
    int boxes;
    int64_t rows;
    int n_in, n_out;
    const int32_t* n_real;
    const void *x, *W, *b, *residual, *grad_y;
    const void* gz;        // kGradX, kGradW: grad_y itself where there is no activation
    int ld_gz;             // elements of its rows: columns behind n_out, if any, hold zeros
    void* out;
    float* shares;         // kGradW: [ranges][n_in * n_out + n_out]; null: the parameters' gradients are written here
    void *grad_W, *grad_b; // (either may be null: not wanted)
    int ranges, want_sums;
    int beside;            // kGradW: launched behind kGradX
    int n_tiles;           // tiles of 128 (kGradW: of its two dimensions, n_tiles x m_tiles) or NT columns
    int m_tiles;
    int stages, resident;  // operand stages; B's chunks stay in shared memory
    int32_t* status;
};

// The backward: one sweep where both widths are at most 64, else three products with gz in memory.  Workspace: [gz | shares];
// ranges: the rows' division (narrow: blocks of the sweep).  direct: no shares; with few rows the blocks of the sweep are
// one cluster and add up among themselves, and the product is one range.
struct BwdLayout { bool narrow, direct; int64_t ld_gz; int m_tiles, ranges; size_t shares, total; };
constexpr int kClusterBlocks = 8;

// Calls with rows > 0 and checked arguments; T: float or __nv_bfloat16.
template <class T> int linear_fwd(LinArgs& a, int act, cudaStream_t st);
template <class T>
int linear_bwd(LinArgs& a, int act, const BwdLayout& L, void* workspace, void* grad_x, void* grad_W, void* grad_b, cudaStream_t st);

}  // namespace layer
}  // namespace e3j
