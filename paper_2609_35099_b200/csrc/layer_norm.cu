// Layer norm with an activation behind it, forward and backward: what radial networks of attention-type equivariant models
// put between a hidden layer and its activation.
//
//   mu, v = mean and variance of a row;  xh = (x - mu) / sqrt(v + eps);  z = xh weight + bias;  y = act(z)
//   backward:  gz = grad_y act'(z);  grad_weight = sum_rows gz xh;  grad_bias = sum_rows gz;  u = gz weight;
//              grad_x = (u - mean(u) - xh mean(u xh)) / sqrt(v + eps)
//
// Both passes are bound by memory and read every row once: a row stays in the registers of the lanes that share it, so mean
// and variance (about the mean: two sums one after the other, no cancellation) cost shuffles, not traffic, and the backward
// forms them again from the x that it has to read anyway instead of having the forward write them.  A row is shared by
// as many lanes as it has 16-byte pieces where that is no more than a warp (64 float32: 16 lanes, two rows a warp), by a
// warp with several pieces a lane, or by several warps.  Rows that do not start on 16 bytes are read by the 4 bytes or by
// the element, lane-strided, so that a lane keeps the same columns, and with them its share of the parameters'
// gradients, in every row.
//
// The parameters' gradients are sums over all rows: every lane adds up its columns over the rows it meets, the warps of a
// block add theirs in order, and sum_shares_kernel adds the blocks' shares in order.  No atomics; the same bits every time.
#include <algorithm>

#include "layer_common.cuh"

namespace e3j {
namespace layer {
namespace {

constexpr int kNormThreads = 256, kNormWarps = kNormThreads / 32;
constexpr int kMostNorm = 4096;   // columns: 8 warps of 16 elements a lane (backward)

struct NormArgs {
    int64_t rows;
    int n, lanes;          // lanes that share a row: a power of two up to 32 (one access a lane), or 32 times a power of two
    float eps, inverse_n;
    int act;
    const void *x, *weight, *bias, *grad_y;
    const int32_t* n_real;
    void* out;             // y, or grad_x (null: not wanted)
    float* shares;         // backward: [blocks][2 n] of grad_weight and grad_bias (null: not wanted)
};

// Sums over the lanes of a row, all of which get them.  Rows of several warps meet in shared memory; consecutive sums use the two
// halves of it in turn, so one barrier a sum is enough.
struct RowSum {
    int lanes, slot, half;
    float2* meet;   // [2][kNormWarps]
    __device__ __forceinline__ float2 operator()(float2 v) {
        for (int o = min(lanes, 32) >> 1; o > 0; o >>= 1) {
            v.x += __shfl_xor_sync(~0u, v.x, o);
            v.y += __shfl_xor_sync(~0u, v.y, o);
        }
        if (lanes > 32) {
            const int warps = lanes >> 5, warp = threadIdx.x >> 5;
            float2* const m = meet + half * kNormWarps;
            half ^= 1;
            if ((threadIdx.x & 31) == 0) m[warp] = v;
            asm volatile("bar.sync %0, %1;" ::"r"(slot + 1), "r"(lanes) : "memory");
            v = m[slot * warps];
            for (int w = 1; w < warps; ++w) { v.x += m[slot * warps + w].x; v.y += m[slot * warps + w].y; }
        }
        return v;
    }
};

// BWD: backward.  V elements an access, NV accesses a lane and row.
template <class T, int V, int NV, bool BWD>
__global__ void __launch_bounds__(kNormThreads, V * NV <= 8 ? 4 : 2) norm_kernel(const NormArgs a) {
    constexpr int E = V * NV;
    constexpr bool kKeep = E <= 8;     // the parameters' columns stay in registers (else they are read from shared memory)
    constexpr bool kAhead = E <= 8;    // the next row is fetched while this one is worked on
    extern __shared__ float params[];  // [weight | bias], later the block's sums
    __shared__ float2 meet[2 * kNormWarps];
    const int n = a.n, lanes = NV == 1 ? min(a.lanes, 32) : a.lanes;
    const int slots = kNormThreads / lanes, slot = threadIdx.x / lanes, lane = threadIdx.x % lanes;
    const T* const x = (const T*)a.x;
    const T* const gy = (const T*)a.grad_y;
    T* const out = (T*)a.out;
    fast::grid_dependency_wait();
    fast::grid_dependency_trigger();
    const int64_t real = real_rows(a.rows, a.n_real);

    auto col = [&](int i) { return (lane + i * lanes) * V; };
    float w[kKeep ? E : 1], b[kKeep ? E : 1];
    if constexpr (kKeep) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const bool in = col(i) < n;
                w[i * V + j] = in && a.weight ? to_float(((const T*)a.weight)[col(i) + j]) : 1.f;
                b[i * V + j] = in && a.bias ? to_float(((const T*)a.bias)[col(i) + j]) : 0.f;
            }
    } else {
        for (int i = threadIdx.x; i < n; i += kNormThreads) {
            params[i] = a.weight ? to_float(((const T*)a.weight)[i]) : 1.f;
            params[n + i] = a.bias ? to_float(((const T*)a.bias)[i]) : 0.f;
        }
        __syncthreads();
    }
    auto weight_at = [&](int i, int j) { if constexpr (kKeep) return w[i * V + j]; else return params[col(i) + j]; };
    auto bias_at = [&](int i, int j) { if constexpr (kKeep) return b[i * V + j]; else return params[n + col(i) + j]; };
    auto fetch = [&](float (&v)[E], const T* from, int64_t row) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float p[V];
            if (row < real && col(i) < n) Pack<T, V>::load(p, from + row * n + col(i));
            else
#pragma unroll
                for (int j = 0; j < V; ++j) p[j] = 0.f;
#pragma unroll
            for (int j = 0; j < V; ++j) v[i * V + j] = p[j];
        }
    };

    RowSum row_sum{lanes, lanes > 32 ? slot : 0, 0, meet};
    float sum_w[BWD ? E : 1], sum_b[BWD ? E : 1];
#pragma unroll
    for (int i = 0; i < (BWD ? E : 1); ++i) sum_w[i] = sum_b[i] = 0.f;
    const int64_t stride = (int64_t)gridDim.x * slots;
    // All lanes of a warp make the same number of turns (the shuffles need them): the turn of a block's first slot counts.
    int64_t row = (int64_t)blockIdx.x * slots + slot;
    float v[E], g[BWD ? E : 1];
    fetch(v, x, row);
    if constexpr (BWD) fetch(g, gy, row);
    for (int64_t first = (int64_t)blockIdx.x * slots; first < a.rows; first += stride, row += stride) {
        float next_v[kAhead ? E : 1], next_g[kAhead && BWD ? E : 1];
        if constexpr (kAhead) {
            fetch(next_v, x, row + stride);
            if constexpr (BWD) fetch(next_g, gy, row + stride);
        }
        float sum = 0.f, square = 0.f;
#pragma unroll
        for (int i = 0; i < E; ++i) sum += v[i];
        const float mean = row_sum(make_float2(sum, 0.f)).x * a.inverse_n;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float d = col(i) < n ? v[i * V + j] - mean : 0.f;
                v[i * V + j] = d;
                square = fmaf(d, d, square);
            }
        // (the accurate root and division: twice a row)
        const float inverse = 1.f / sqrtf(fmaf(row_sum(make_float2(square, 0.f)).x, a.inverse_n, a.eps));
        float z[E];
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                v[i * V + j] *= inverse;
                const bool in = kKeep || col(i) < n;
                z[i * V + j] = in ? fmaf(v[i * V + j], weight_at(i, j), bias_at(i, j)) : 0.f;
            }
        if constexpr (!BWD) {
            activate(z, a.act);
        } else {
            times_slope(g, z, a.act);
            float2 means = make_float2(0.f, 0.f);
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const int k = i * V + j;
                    sum_b[k] += g[k];   // (zero in padding rows and behind the last column)
                    sum_w[k] = fmaf(g[k], v[k], sum_w[k]);
                    const bool in = kKeep || col(i) < n;
                    g[k] *= in ? weight_at(i, j) : 0.f;
                    means.x += g[k];
                    means.y = fmaf(g[k], v[k], means.y);
                }
            means = row_sum(means);
            means.x *= a.inverse_n;
            means.y *= a.inverse_n;
#pragma unroll
            for (int k = 0; k < E; ++k) z[k] = (g[k] - fmaf(v[k], means.y, means.x)) * inverse;
        }
        if (row < a.rows && out) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                float p[V];
#pragma unroll
                for (int j = 0; j < V; ++j) p[j] = row < real ? z[i * V + j] : 0.f;
                if (col(i) < n) Pack<T, V>::store(out + row * n + col(i), p);
            }
        }
        if constexpr (kAhead) {
#pragma unroll
            for (int i = 0; i < E; ++i) v[i] = next_v[i];
            if constexpr (BWD)
#pragma unroll
                for (int i = 0; i < E; ++i) g[i] = next_g[i];
        } else {
            fetch(v, x, row + stride);
            if constexpr (BWD) fetch(g, gy, row + stride);
        }
    }
    if constexpr (BWD) {
        if (!a.shares) return;
        // the rows of a warp first, then the block's warps (or its slots of several warps) in order
        if (lanes < 32)
#pragma unroll
            for (int i = 0; i < E; ++i)
                for (int o = 16; o >= lanes; o >>= 1) {
                    sum_w[i] += __shfl_xor_sync(~0u, sum_w[i], o);
                    sum_b[i] += __shfl_xor_sync(~0u, sum_b[i], o);
                }
        const int turns = lanes <= 32 ? kNormWarps : slots, turn = lanes <= 32 ? (int)threadIdx.x >> 5 : slot;
        const bool speaks = lanes >= 32 || (threadIdx.x & 31) < lanes;
        for (int t = 0; t < turns; ++t) {
            __syncthreads();   // (the first: nobody reads the parameters any more)
            if (t == turn && speaks)
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int j = 0; j < V; ++j)
                        if (col(i) < n) {
                            float *pw = params + col(i) + j, *pb = pw + n;
                            *pw = t == 0 ? sum_w[i * V + j] : *pw + sum_w[i * V + j];
                            *pb = t == 0 ? sum_b[i * V + j] : *pb + sum_b[i * V + j];
                        }
        }
        __syncthreads();
        float* const to = a.shares + (int64_t)blockIdx.x * 2 * n;
        for (int i = threadIdx.x; i < 2 * n; i += kNormThreads) to[i] = params[i];
    }
}

// What a call runs on: V elements an access, NV accesses a lane, lanes a row.
struct NormShape { int v, nv, lanes, blocks; };

// Elements a lane: up to 32 in the forward, up to 16 in the backward, which holds four such sets.
NormShape norm_shape(int64_t rows, int n, int widest, bool bwd) {
    NormShape s{};
    s.v = widest;
    const int most = bwd ? 16 : 32;
    const int pieces = (n + s.v - 1) / s.v;
    s.lanes = 1;
    while (s.lanes < 32 && s.lanes < pieces) s.lanes *= 2;
    s.nv = 1;
    while ((int64_t)s.lanes * s.nv < pieces) {
        if (s.v * s.nv < most) s.nv *= 2;
        else s.lanes *= 2;
    }
    const int64_t per_turn = kNormThreads / s.lanes;
    const int64_t resident = (int64_t)sm_count() * (s.v * s.nv <= 8 ? 4 : 2);
    s.blocks = (int)std::min<int64_t>((rows + per_turn - 1) / per_turn, resident);
    return s;
}

// The widest access that every row's start allows.
template <class T> int widest_access(int n, const void* const (&arrays)[3]) {
    uintptr_t all = (uintptr_t)n * sizeof(T);
    for (const void* p : arrays) all |= (uintptr_t)p;
    if ((all & 15u) == 0) return 16 / (int)sizeof(T);
    return sizeof(T) == 2 && (all & 3u) == 0 ? 2 : 1;
}

template <class T, int V, int NV, bool BWD> int launch_norm(const NormArgs& a, const NormShape& s, cudaStream_t st) {
    return launch_dependent(norm_kernel<T, V, NV, BWD>, dim3((unsigned)s.blocks), dim3(kNormThreads),
                            sizeof(float) * 2 * (size_t)a.n, st, a);
}
template <class T, int V, bool BWD> int launch_norm_nv(const NormArgs& a, const NormShape& s, cudaStream_t st) {
    switch (s.nv) {
        case 1: return launch_norm<T, V, 1, BWD>(a, s, st);
        case 2: return launch_norm<T, V, 2, BWD>(a, s, st);
        case 4: if constexpr (V * 4 <= (BWD ? 16 : 32)) return launch_norm<T, V, 4, BWD>(a, s, st); break;
        case 8: if constexpr (V * 8 <= (BWD ? 16 : 32)) return launch_norm<T, V, 8, BWD>(a, s, st); break;
        case 16: if constexpr (V * 16 <= (BWD ? 16 : 32)) return launch_norm<T, V, 16, BWD>(a, s, st); break;
        case 32: if constexpr (V * 32 <= (BWD ? 16 : 32)) return launch_norm<T, V, 32, BWD>(a, s, st); break;
    }
    return E3J_ERR_UNSUPPORTED;
}
template <class T, bool BWD> int norm(NormArgs a, const NormShape& s, cudaStream_t st) {
    a.lanes = s.lanes;
    if constexpr (sizeof(T) == 2) {
        if (s.v == 8) return launch_norm_nv<T, 8, BWD>(a, s, st);
        if (s.v == 2) return launch_norm_nv<T, 2, BWD>(a, s, st);
    } else {
        if (s.v == 4) return launch_norm_nv<T, 4, BWD>(a, s, st);
    }
    return launch_norm_nv<T, 1, BWD>(a, s, st);
}

template <class T>
int norm_fwd(NormArgs& a, cudaStream_t st) {
    return norm<T, false>(a, norm_shape(a.rows, a.n, widest_access<T>(a.n, {a.x, a.out, nullptr}), false), st);
}
template <class T>
int norm_bwd(NormArgs& a, void* grad_weight, void* grad_bias, cudaStream_t st) {
    const NormShape s = norm_shape(a.rows, a.n, widest_access<T>(a.n, {a.x, a.grad_y, a.out}), true);
    if (!grad_weight && !grad_bias) a.shares = nullptr;
    if (int rc = norm<T, true>(a, s, st)) return rc;
    if (!a.shares) return E3J_OK;
    return sum_shares<T>(s.blocks, a.n, a.n, a.shares, (T*)grad_weight, (T*)grad_bias, st);
}

int norm_args_status(int64_t rows, int n, int dtype, double eps, int act) {
    if (rows < 0 || n < 1 || !(eps >= 0.0) || dtype < E3J_F32 || dtype > E3J_BF16 || act < E3J_ACT_NONE || act > E3J_ACT_GELU)
        return E3J_ERR_INVALID_ARG;
    return n > kMostNorm || rows >= (1ll << 31) - 1 ? E3J_ERR_UNSUPPORTED : E3J_OK;
}

}  // namespace
}  // namespace layer
}  // namespace e3j

using namespace e3j;
using namespace e3j::layer;

extern "C" {

int e3j_layer_norm_fwd(int dtype, int64_t rows, int n, const void* x, const void* weight, const void* bias, double eps, int act,
                       const int32_t* n_real, void* y, void* stream) {
    if (int rc = norm_args_status(rows, n, dtype, eps, act)) return rc;
    if (rows == 0) return E3J_OK;
    if (!x || !y) return E3J_ERR_INVALID_ARG;
    const uintptr_t odd = dtype == E3J_F32 ? 3u : 1u;
    if (((uintptr_t)x | (uintptr_t)weight | (uintptr_t)bias | (uintptr_t)y) & odd) return E3J_ERR_INVALID_ARG;
    NormArgs a{};
    a.rows = rows; a.n = n; a.eps = (float)eps; a.inverse_n = 1.f / (float)n; a.act = act;
    a.x = x; a.weight = weight; a.bias = bias; a.n_real = n_real; a.out = y;
    return dtype == E3J_F32 ? norm_fwd<float>(a, (cudaStream_t)stream) : norm_fwd<bf16>(a, (cudaStream_t)stream);
}

size_t e3j_layer_norm_bwd_workspace_bytes(int dtype, int64_t rows, int n) {
    if (norm_args_status(rows, n, dtype, 0.0, E3J_ACT_NONE) != E3J_OK) return 0;
    // (an access may be narrower than the width allows, where an array does not start on its boundary: more blocks)
    size_t most = 0;
    for (int v : {1, 2, 4, 8}) most = std::max(most, (size_t)norm_shape(rows, n, v, true).blocks);
    return align_up(std::max<size_t>(most, 1) * 2 * n * sizeof(float), 256);
}

int e3j_layer_norm_bwd(int dtype, int64_t rows, int n, const void* x, const void* weight, const void* bias, const void* grad_y,
                       double eps, int act, const int32_t* n_real, void* grad_x, void* grad_weight, void* grad_bias,
                       void* workspace, size_t workspace_bytes, void* stream) {
    if (int rc = norm_args_status(rows, n, dtype, eps, act)) return rc;
    cudaStream_t st = (cudaStream_t)stream;
    const size_t size = dtype == E3J_F32 ? 4 : 2;
    const uintptr_t arrays = (uintptr_t)x | (uintptr_t)weight | (uintptr_t)bias | (uintptr_t)grad_y | (uintptr_t)grad_x |
                             (uintptr_t)grad_weight | (uintptr_t)grad_bias;
    if (arrays & (size - 1)) return E3J_ERR_INVALID_ARG;
    if (rows == 0) {   // sums over no rows
        if (grad_weight) E3J_CUDA_TRY(cudaMemsetAsync(grad_weight, 0, size * n, st));
        if (grad_bias) E3J_CUDA_TRY(cudaMemsetAsync(grad_bias, 0, size * n, st));
        return E3J_OK;
    }
    if (!x || !grad_y) return E3J_ERR_INVALID_ARG;
    if (!grad_x && !grad_weight && !grad_bias) return E3J_OK;
    if ((grad_weight || grad_bias) && (!workspace || ((uintptr_t)workspace & 255u) ||
                                       workspace_bytes < e3j_layer_norm_bwd_workspace_bytes(dtype, rows, n)))
        return E3J_ERR_WORKSPACE;
    NormArgs a{};
    a.rows = rows; a.n = n; a.eps = (float)eps; a.inverse_n = 1.f / (float)n; a.act = act;
    a.x = x; a.weight = weight; a.bias = bias; a.grad_y = grad_y; a.n_real = n_real; a.out = grad_x;
    a.shares = (float*)workspace;
    return dtype == E3J_F32 ? norm_bwd<float>(a, grad_weight, grad_bias, st) : norm_bwd<bf16>(a, grad_weight, grad_bias, st);
}

}  // extern "C"
