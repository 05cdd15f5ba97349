// Layer norm with an activation behind it, forward and backward: what radial networks of attention-type equivariant models
// put between a hidden layer and its activation.
//
//   mu, v = mean and variance of a row;  xh = (x - mu) / sqrt(v + eps);  z = xh weight + bias;  y = act(z)
//   backward:  gz = grad_y act'(z);  grad_weight = sum_rows gz xh;  grad_bias = sum_rows gz;  u = gz weight;
//              grad_x = (u - mean(u) - xh mean(u xh)) / sqrt(v + eps)
//
// Both passes are bound by memory and read every row once: a row stays in the registers of the lanes that share it, so mean
// and variance (about the mean: two sums one after the other, no cancellation) cost shuffles, not traffic, and the backward
// forms them again from the x that it has to read anyway instead of having the forward write them.  A lane has 8 elements of a
// row: with fewer, what a row costs once (the sums' shuffles, the root) bounds narrow rows.  So a row of 64 is shared by 8 lanes, four
// rows a warp; beyond 256 columns it is whole warps, up to eight of them a row, and 16 elements where the registers hold them
// (sixteen_elements), beyond 2048 columns anyway.  Arithmetic on pairs
// (packed float32 instructions), since with 2-byte elements the instructions, not the memory, come first.
//
// The parameters' gradients are sums over all rows: every lane adds up its columns over the rows it meets, the warps of a
// block add theirs in order, and sum_shares_kernel adds the blocks' shares in order.  No atomics; the same bits every time.
#include <cooperative_groups.h>

#include <algorithm>

#include "layer_common.cuh"

namespace e3j {
namespace layer {
namespace {

constexpr int kNormThreads = 256, kNormWarps = kNormThreads / 32;
constexpr int kClusterBlocks = 8, kClusterTurns = 6;   // backward of few rows
constexpr int kMostNorm = 4096;   // columns: 256 lanes of 16 elements

struct NormArgs {
    int64_t rows;
    int n, lanes;          // lanes that share a row: a power of two
    float eps, inverse_n;
    int act;
    const void *x, *weight, *bias, *grad_y;
    const int32_t* n_real;
    void* out;             // y, or grad_x (null: not wanted)
    float* shares;         // backward: [blocks][2 n] of grad_weight and grad_bias; null: the blocks, one cluster, add them up
    void *grad_weight, *grad_bias;   // (either may be null: not wanted)
};

// Sums over the lanes of a row (LANES; 0: several warps), all of which get them.  Rows of several warps meet in shared memory;
// consecutive sums use the two halves of it in turn, so one barrier a sum is enough.
template <int LANES> struct RowSum {
    int lanes, slot, half;
    float2* meet;   // [2][kNormWarps]
    __device__ __forceinline__ void within_warp(float& v) {
#pragma unroll
        for (int o = (LANES ? LANES : 32) >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    }
    __device__ __forceinline__ float2 operator()(float2 v) {
        within_warp(v.x);
        within_warp(v.y);
        if constexpr (LANES == 0) {
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
    __device__ __forceinline__ float operator()(float v) { return (*this)(make_float2(v, 0.f)).x; }
};

// Whether lanes have 16 elements of rows beyond 256 columns, not of those beyond 2048 alone: fewer lanes to sum over.
__host__ __device__ constexpr bool sixteen_elements(int size, bool vector, bool ragged, bool bwd) { return !bwd || (size == 2 && vector && !ragged); }
// Blocks an SM: as many as the registers allow (nearly) without spilling.
__host__ __device__ constexpr int norm_blocks(int v, int each, bool ragged, bool bwd) {
    return v == 1 ? (each == 8 && !bwd ? 2 : 1)
         : each == 8 ? (!bwd ? (ragged ? 3 : 4) : v == 4 || ragged ? 2 : 3)
         : v == 4 ? (bwd ? 1 : 2) : (bwd ? (ragged ? 1 : 2) : ragged ? 2 : 3);
}

// BWD: backward.  V elements an access, EACH a lane and row; LANES lanes a row (0: a.lanes of them, whole warps).
// RAGGED: rows do not start on 16 bytes.  A row's lanes then count from the 16-byte boundary before its start, `shift` columns to
// the left of it; the grid's stride is a multiple of V rows, so a slot's rows all have the same shift and its lanes keep
// their columns.  Accesses that reach over an end of the row go element by element.
template <class T, int V, int EACH, int LANES, bool RAGGED, bool BWD>
__global__ void __launch_bounds__(kNormThreads, norm_blocks(V, EACH, RAGGED, BWD)) norm_kernel(const NormArgs a) {
    constexpr int NV = EACH / V;
    using P = Pack<T, V>;
    constexpr int H = P::kPairs, E2 = NV * H;   // pairs of an access, of a lane
    extern __shared__ float block_sums[];       // backward: [warps or slots][2][n], the first row then the block's
    __shared__ float2 meet[2 * kNormWarps];
    const int n = a.n, lanes = LANES ? LANES : a.lanes;
    const int slots = kNormThreads / lanes, slot = threadIdx.x / lanes, lane = threadIdx.x % lanes;
    const T* const x = (const T*)a.x;
    const T* const gy = (const T*)a.grad_y;
    T* const out = (T*)a.out;
    fast::grid_dependency_wait();
    fast::grid_dependency_trigger();
    const int64_t real = real_rows(a.rows, a.n_real);
    const int64_t stride = (int64_t)gridDim.x * slots;
    int64_t row = (int64_t)blockIdx.x * slots + slot;

    const int shift = RAGGED ? (int)(row * n % V) : 0;
    auto col = [&](int i) { return (lane + i * lanes) * V - shift; };
    auto whole = [&](int i) { return RAGGED ? col(i) >= 0 && col(i) + V <= n : col(i) < n; };
    auto inside = [&](int c) { return RAGGED ? c >= 0 && c < n : c < n; };
    // access i of a row from its elements, those outside the row 0
    auto piecewise = [&](const T* at, int i) {
        float2 v[H];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float f = inside(col(i) + j) ? to_float(at[col(i) + j]) : 0.f;
            if (j & 1) v[j / 2].y = f;
            else v[j / 2] = make_float2(f, 0.f);
        }
        return P::from(v);
    };
    const int64_t all = a.rows * n;
    struct Part { typename P::Raw r[NV]; };     // a lane's part of a row, as it lies in memory
    auto fetch = [&](Part& p, const T* from, int64_t r) {
        const T* const at = from + r * n;
        if (r < real) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                // (an access over an end of the row takes in some of the next row, or of the one before; not over the array's)
                if (whole(i) || (RAGGED && col(i) < n && r * n + col(i) + V <= all)) p.r[i] = P::fetch(at + col(i));
                else if (RAGGED && col(i) < n) p.r[i] = piecewise(at, i);
                else p.r[i] = P::none();
            }
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i) p.r[i] = P::none();
        }
    };
    Part masks;   // RAGGED: ones in the bits of the columns inside the row
    if constexpr (RAGGED)
#pragma unroll
        for (int i = 0; i < NV; ++i) masks.r[i] = P::ones([&](int j) { return inside(col(i) + j); });
    // this lane's columns of the parameters; columns outside the row: 0
    Part w, b;
    {
        float2 ones[H];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
#pragma unroll
            for (int j = 0; j < H; ++j) ones[j] = make_float2(inside(col(i) + 2 * j) ? 1.f : 0.f, inside(col(i) + 2 * j + 1) ? 1.f : 0.f);
            w.r[i] = a.weight ? piecewise((const T*)a.weight, i) : P::from(ones);
            b.r[i] = a.bias ? piecewise((const T*)a.bias, i) : P::none();
        }
    }

    RowSum<LANES> row_sum{lanes, slot, 0, meet};
    float2 sum_w[BWD ? E2 : 1], sum_b[BWD ? E2 : 1];
#pragma unroll
    for (int k = 0; k < (BWD ? E2 : 1); ++k) sum_w[k] = sum_b[k] = make_float2(0.f, 0.f);
    // the next row is on its way while one is worked on (two or three rows ahead: slower, 160 900 x 64 float32 forward, the same arrays over and
    // over, some of them in L2, 12.0 -> 14.9 us)
    Part next_x, next_g;
    fetch(next_x, x, row);
    if constexpr (BWD) fetch(next_g, gy, row);
    // All lanes of a block make the same number of turns (the shuffles need them): its first slot's row counts.
    for (int64_t first = (int64_t)blockIdx.x * slots; first < a.rows; first += stride, row += stride) {
        if (first >= real) {   // (the whole block's rows)
            if (row < a.rows && out)
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    T* const at = out + row * n + col(i);
                    if (whole(i)) P::store(at, P::none());
                    else if constexpr (RAGGED) P::store_inside(at, P::none(), masks.r[i]);
                }
            continue;
        }
        float2 v[E2], g[BWD ? E2 : 1];
        if constexpr (RAGGED) {   // (without what an access took in from outside the row)
            P::mask(next_x.r, masks);
            if constexpr (BWD) P::mask(next_g.r, masks);
        }
#pragma unroll
        for (int k = 0; k < E2; ++k) {
            v[k] = P::pair(next_x.r[k / H], k % H);
            if constexpr (BWD) g[k] = P::pair(next_g.r[k / H], k % H);
        }
        fetch(next_x, x, row + stride);
        if constexpr (BWD) fetch(next_g, gy, row + stride);
        float2 sum = v[0];
#pragma unroll
        for (int k = 1; k < E2; ++k) sum = __fadd2_rn(sum, v[k]);
        const float mean = row_sum(sum.x + sum.y) * a.inverse_n;
        float2 square = make_float2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            // (outside the row v becomes -mean, which nothing but this sum sees: weight, bias and grad_y are 0 there)
            if (whole(i)) {
#pragma unroll
                for (int j = 0; j < H; ++j) {
                    v[i * H + j] = V == 1 ? make_float2(v[i * H].x - mean, 0.f) : __fadd2_rn(v[i * H + j], both(-mean));
                    square = __ffma2_rn(v[i * H + j], v[i * H + j], square);
                }
            } else if (RAGGED) {   // (without, there is nothing but zeros here)
#pragma unroll
                for (int j = 0; j < H; ++j) {
                    v[i * H + j] = __fadd2_rn(v[i * H + j], both(-mean));
                    if (inside(col(i) + 2 * j)) square.x = fmaf(v[i * H + j].x, v[i * H + j].x, square.x);
                    if (inside(col(i) + 2 * j + 1)) square.y = fmaf(v[i * H + j].y, v[i * H + j].y, square.y);
                }
            }
        }
        const float variance = row_sum(square.x + square.y) * a.inverse_n;
        // (a padding row is zero throughout, also with eps = 0)
        const float inverse = row < real ? rsqrtf(variance + a.eps) : 0.f;
        const float2 inverse2 = make_float2(inverse, inverse);
        float2 z[E2];
#pragma unroll
        for (int k = 0; k < E2; ++k) {
            v[k] = __fmul2_rn(v[k], inverse2);
            z[k] = __ffma2_rn(v[k], P::pair(w.r[k / H], k % H), P::pair(b.r[k / H], k % H));
        }
        if constexpr (!BWD) {
            activate<T>(z, a.act);
        } else {
            times_slope<T>(g, z, a.act);
            float2 mean_u = make_float2(0.f, 0.f), mean_uv = mean_u;
#pragma unroll
            for (int k = 0; k < E2; ++k) {   // (g is zero in padding rows and outside the row)
                sum_b[k] = __fadd2_rn(sum_b[k], g[k]);
                sum_w[k] = __ffma2_rn(g[k], v[k], sum_w[k]);
                g[k] = __fmul2_rn(g[k], P::pair(w.r[k / H], k % H));
                mean_u = __fadd2_rn(mean_u, g[k]);
                mean_uv = __ffma2_rn(g[k], v[k], mean_uv);
            }
            const float2 means = row_sum(make_float2(mean_u.x + mean_u.y, mean_uv.x + mean_uv.y));
            const float2 m0 = make_float2(-means.x * a.inverse_n, -means.x * a.inverse_n);
            const float2 m1 = make_float2(-means.y * a.inverse_n, -means.y * a.inverse_n);
#pragma unroll
            for (int k = 0; k < E2; ++k) z[k] = __fmul2_rn(__fadd2_rn(g[k], __ffma2_rn(v[k], m1, m0)), inverse2);
        }
        if (row < a.rows && out) {
            T* const at = out + row * n;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                float2 o[H];
#pragma unroll
                for (int j = 0; j < H; ++j) o[j] = z[i * H + j];
                const typename P::Raw r = row < real ? P::from(o) : P::none();
                if (whole(i)) P::store(at + col(i), r);
                else if constexpr (RAGGED) P::store_inside(at + col(i), r, masks.r[i]);
            }
        }
    }
    if constexpr (BWD) {
        if (!a.grad_weight && !a.grad_bias) return;
        // the rows of a warp first where they have the same columns, then what is left in order: a warp's slots, the block's warps
        constexpr bool kTogether = !RAGGED && LANES > 0 && LANES < 32;
        if constexpr (kTogether)
#pragma unroll
            for (int k = 0; k < E2; ++k)
#pragma unroll
                for (int o = 16; o >= LANES; o >>= 1) {
                    sum_w[k].x += __shfl_xor_sync(~0u, sum_w[k].x, o);
                    sum_w[k].y += __shfl_xor_sync(~0u, sum_w[k].y, o);
                    sum_b[k].x += __shfl_xor_sync(~0u, sum_b[k].x, o);
                    sum_b[k].y += __shfl_xor_sync(~0u, sum_b[k].y, o);
                }
        // every warp (or slot of several warps) leaves its sums in a row of its own
        const int rows_of_sums = LANES ? kNormWarps : slots;
        float* const mine = block_sums + (LANES ? (int)threadIdx.x >> 5 : slot) * 2 * n;
        if constexpr (RAGGED && LANES > 0 && LANES < 32) {   // (a warp's slots have other columns: one after another)
            for (int i = threadIdx.x & 31; i < 2 * n; i += 32) mine[i] = 0.f;
            __syncwarp();
        }
        const int speakers = RAGGED && LANES > 0 && LANES < 32 ? 32 / lanes : 1;
        for (int s = 0; s < speakers; ++s) {
            if (LANES == 0 || (int)(threadIdx.x & 31) / lanes == s)
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int j = 0; j < V; ++j)
                        if (inside(col(i) + j)) {
                            const float2 sw = sum_w[i * H + j / 2], sb = sum_b[i * H + j / 2];
                            float *pw = mine + col(i) + j, *pb = pw + n;
                            *pw = (speakers > 1 ? *pw : 0.f) + (j & 1 ? sw.y : sw.x);
                            *pb = (speakers > 1 ? *pb : 0.f) + (j & 1 ? sb.y : sb.x);
                        }
            __syncwarp();
        }
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * n; i += kNormThreads) {
            float sum = block_sums[i];
            for (int r = 1; r < rows_of_sums; ++r) sum += block_sums[r * 2 * n + i];
            block_sums[i] = sum;
        }
        __syncthreads();
        if (a.shares) {
            float* const to = a.shares + (int64_t)blockIdx.x * 2 * n;
            for (int i = threadIdx.x; i < 2 * n; i += kNormThreads) to[i] = block_sums[i];
        } else {   // few rows: in the order of the cluster's blocks
            const auto cluster = cooperative_groups::this_cluster();
            cluster.sync();
            for (int i = blockIdx.x * kNormThreads + threadIdx.x; i < 2 * n; i += gridDim.x * kNormThreads) {
                float theirs[kClusterBlocks], sum = 0.f;   // (all on their way before the first is added)
#pragma unroll
                for (int r = 0; r < kClusterBlocks; ++r) theirs[r] = r < (int)gridDim.x ? cluster.map_shared_rank(block_sums, r)[i] : 0.f;
#pragma unroll
                for (int r = 0; r < kClusterBlocks; ++r) sum += theirs[r];
                if (i < n && a.grad_weight) ((T*)a.grad_weight)[i] = from_float<T>(sum);
                if (i >= n && a.grad_bias) ((T*)a.grad_bias)[i - n] = from_float<T>(sum);
            }
            cluster.sync();   // (nobody leaves while others read)
        }
    }
}

// What a call runs on.  16-byte accesses where the arrays start on 16 bytes, element by element elsewhere and in narrow rows that do
// not (32 columns or fewer: little data, and sums slot by slot would take longer than the rows).
struct NormShape { int vector, ragged, each, lanes, blocks, direct; };

NormShape norm_shape(int64_t rows, int n, int size, bool bwd, bool aligned) {
    NormShape s{};
    const int v = 16 / size;
    s.ragged = aligned && n % v != 0 && n > 32 && n + v - 1 <= 16 * kNormThreads;
    s.vector = aligned && (n % v == 0 || s.ragged);
    const int width = n + (s.ragged ? v - 1 : 0);
    s.each = width > 8 * kNormThreads || (width > 256 && sixteen_elements(size, s.vector, s.ragged, bwd)) ? 16 : 8;
    s.lanes = 1;
    while (s.lanes * s.each < width) s.lanes *= 2;
    if (s.each == 16) s.lanes = std::max(s.lanes, 32);
    const int64_t per_turn = kNormThreads / s.lanes;
    const int64_t resident = (int64_t)sm_count() * norm_blocks(s.vector ? v : 1, s.each, s.ragged, bwd);
    s.blocks = (int)std::min<int64_t>((rows + per_turn - 1) / per_turn, resident);
    // Few rows, backward: one cluster, whose blocks take up to kClusterTurns turns, and no second kernel for the sums.  What counts is the host,
    // which calls of this size wait for: 9.1 us a call where two kernels are 13.1, as long as the cluster is not slower than that (on
    // the device, cluster and two kernels: 1536 x 64 float32, 6 turns, 6.5 and 4.4 us; 384 x 512 bfloat16, 6 turns, 11.8 and 6.7; 192 x 385
    // 13.9 and 6.6; with 12 turns 760 x 512 18.6 and 6.9).
    s.direct = bwd && rows <= kClusterBlocks * kClusterTurns * per_turn;
    if (s.direct) s.blocks = std::min(s.blocks, kClusterBlocks);
    const int step = (int)std::max<int64_t>(v / per_turn, 1);   // (ragged rows: the stride is a multiple of v rows)
    if (s.ragged) s.blocks = (s.blocks + step - 1) / step * step;
    return s;
}

template <class T, int V, int EACH, int LANES, bool RAGGED, bool BWD> int launch_norm(const NormArgs& a, const NormShape& s, cudaStream_t st) {
    return launch_cluster(norm_kernel<T, V, EACH, LANES, RAGGED, BWD>, s.blocks, s.direct ? s.blocks : 1, kNormThreads,
                          BWD ? sizeof(float) * 2 * (size_t)a.n * (LANES ? kNormWarps : kNormThreads / s.lanes) : 0, st, a);   // (32 KB at most)
}
template <class T, int V, bool RAGGED, bool BWD> int launch_norm_lanes(const NormArgs& a, const NormShape& s, cudaStream_t st) {
    constexpr bool kSixteen = sixteen_elements(sizeof(T), V > 1, RAGGED, BWD);   // (else 16 elements are more than 2048 columns: 256 lanes)
    if constexpr (kSixteen)
        if (s.each == 16 && s.lanes == 32) return launch_norm<T, V, 16, 32, RAGGED, BWD>(a, s, st);
    if (s.each == 16) return launch_norm<T, V, 16, 0, RAGGED, BWD>(a, s, st);
    if constexpr (!RAGGED) {   // (more than 32 columns: 8 lanes and more)
        if (s.lanes == 1) return launch_norm<T, V, 8, 1, RAGGED, BWD>(a, s, st);
        if (s.lanes == 2) return launch_norm<T, V, 8, 2, RAGGED, BWD>(a, s, st);
        if (s.lanes == 4) return launch_norm<T, V, 8, 4, RAGGED, BWD>(a, s, st);
    }
    if (s.lanes == 8) return launch_norm<T, V, 8, 8, RAGGED, BWD>(a, s, st);
    if (s.lanes == 16) return launch_norm<T, V, 8, 16, RAGGED, BWD>(a, s, st);
    if constexpr (kSixteen) return launch_norm<T, V, 8, 32, RAGGED, BWD>(a, s, st);   // (8 elements are up to 256 columns)
    else return s.lanes == 32 ? launch_norm<T, V, 8, 32, RAGGED, BWD>(a, s, st) : launch_norm<T, V, 8, 0, RAGGED, BWD>(a, s, st);
}
template <class T, bool BWD> int norm(NormArgs a, const NormShape& s, cudaStream_t st) {
    a.lanes = s.lanes;
    constexpr int V = 16 / (int)sizeof(T);
    if (s.ragged) return launch_norm_lanes<T, V, true, BWD>(a, s, st);
    return s.vector ? launch_norm_lanes<T, V, false, BWD>(a, s, st) : launch_norm_lanes<T, 1, false, BWD>(a, s, st);
}
inline bool on_16_bytes(const void* p, const void* q, const void* r) { return (((uintptr_t)p | (uintptr_t)q | (uintptr_t)r) & 15u) == 0; }

template <class T>
int norm_fwd(NormArgs& a, cudaStream_t st) {
    return norm<T, false>(a, norm_shape(a.rows, a.n, sizeof(T), false, on_16_bytes(a.x, a.out, nullptr)), st);
}
template <class T>
int norm_bwd(NormArgs& a, void* grad_weight, void* grad_bias, cudaStream_t st) {
    const NormShape s = norm_shape(a.rows, a.n, sizeof(T), true, on_16_bytes(a.x, a.grad_y, a.out));
    a.grad_weight = grad_weight;
    a.grad_bias = grad_bias;
    if (s.direct) a.shares = nullptr;
    if (int rc = norm<T, true>(a, s, st)) return rc;
    if (s.direct || (!grad_weight && !grad_bias)) return E3J_OK;
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
    if ((uintptr_t)n_real & 3u) return E3J_ERR_INVALID_ARG;
    NormArgs a{};
    a.rows = rows; a.n = n; a.eps = (float)eps; a.inverse_n = 1.f / (float)n; a.act = act;
    a.x = x; a.weight = weight; a.bias = bias; a.n_real = n_real; a.out = y;
    return dtype == E3J_F32 ? norm_fwd<float>(a, (cudaStream_t)stream) : norm_fwd<bf16>(a, (cudaStream_t)stream);
}

size_t e3j_layer_norm_bwd_workspace_bytes(int dtype, int64_t rows, int n) {
    if (norm_args_status(rows, n, dtype, 0.0, E3J_ACT_NONE) != E3J_OK) return 0;
    const int size = dtype == E3J_F32 ? 4 : 2;
    size_t most = 0;   // (arrays that do not start on 16 bytes may have another number of blocks)
    for (bool aligned : {false, true}) {
        const NormShape s = norm_shape(rows, n, size, true, aligned);
        if (!s.direct) most = std::max<size_t>(most, s.blocks);
    }
    return align_up(most * 2 * n * sizeof(float), 256);
}

int e3j_layer_norm_bwd(int dtype, int64_t rows, int n, const void* x, const void* weight, const void* bias, const void* grad_y,
                       double eps, int act, const int32_t* n_real, void* grad_x, void* grad_weight, void* grad_bias,
                       void* workspace, size_t workspace_bytes, void* stream) {
    if (int rc = norm_args_status(rows, n, dtype, eps, act)) return rc;
    cudaStream_t st = (cudaStream_t)stream;
    const size_t size = dtype == E3J_F32 ? 4 : 2;
    const uintptr_t arrays = (uintptr_t)x | (uintptr_t)weight | (uintptr_t)bias | (uintptr_t)grad_y | (uintptr_t)grad_x |
                             (uintptr_t)grad_weight | (uintptr_t)grad_bias;
    if ((arrays & (size - 1)) || ((uintptr_t)n_real & 3u)) return E3J_ERR_INVALID_ARG;
    if (rows == 0) {   // sums over no rows
        if (grad_weight) E3J_CUDA_TRY(cudaMemsetAsync(grad_weight, 0, size * n, st));
        if (grad_bias) E3J_CUDA_TRY(cudaMemsetAsync(grad_bias, 0, size * n, st));
        return E3J_OK;
    }
    if (!x || !grad_y) return E3J_ERR_INVALID_ARG;
    if (!grad_x && !grad_weight && !grad_bias) return E3J_OK;
    const size_t need = grad_weight || grad_bias ? e3j_layer_norm_bwd_workspace_bytes(dtype, rows, n) : 0;
    if (need > 0 && (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < need)) return E3J_ERR_WORKSPACE;
    NormArgs a{};
    a.rows = rows; a.n = n; a.eps = (float)eps; a.inverse_n = 1.f / (float)n; a.act = act;
    a.x = x; a.weight = weight; a.bias = bias; a.grad_y = grad_y; a.n_real = n_real; a.out = grad_x;
    a.shares = (float*)workspace;
    return dtype == E3J_F32 ? norm_bwd<float>(a, grad_weight, grad_bias, st) : norm_bwd<bf16>(a, grad_weight, grad_bias, st);
}

}  // extern "C"
