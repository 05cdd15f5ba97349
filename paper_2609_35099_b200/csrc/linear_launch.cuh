// Launches of linear_kernels.cuh for one type of the layer's tensors: included by linear_f32.cu and linear_bf16.cu.
#pragma once
#include <algorithm>
#include <atomic>

#include "linear.hpp"
#include "linear_bwd_narrow.cuh"
#include "linear_kernels.cuh"
#include "tensor_map.hpp"

namespace e3j {
namespace layer {

constexpr size_t kSmemOfBlock = 227 * 1024;

// Lets a kernel have that much dynamic shared memory on the current device (once: a bit per device).
template <class K> int allow_smem(K kernel, size_t bytes, std::atomic<uint64_t>& allowed) {
    int dev = 0;
    E3J_CUDA_TRY(cudaGetDevice(&dev));
    if (dev < 0 || dev >= 64) return E3J_ERR_UNSUPPORTED;
    if (!(allowed.load(std::memory_order_relaxed) >> dev & 1)) {
        E3J_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
        allowed.fetch_or(1ull << dev, std::memory_order_relaxed);
    }
    return E3J_OK;
}

// Tensor map of a bfloat16 matrix whose rows start on 16 bytes, fetched in boxes of 128 x 64 as operand images; false where the driver
// has no encoder.
inline bool box_map(CUtensorMap* map, const void* base, int64_t rows, int columns) {
    const EncodeTiled encode = tensor_map_encoder();
    const cuuint64_t dims[2] = {(cuuint64_t)columns, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)columns * 2};
    const cuuint32_t box[2] = {kChunk, kTileRows}, elem[2] = {1, 1};
    return encode && encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <Product P, class T, class G, int NT, int ACT, bool VA, bool VO, Chains CHAINS = kOne>
struct Launch {
    using L = LinTile<P, T, G, NT, VA, VO, CHAINS>;
    static constexpr auto kernel = linear_kernel<P, T, G, NT, ACT, VA, VO, CHAINS>;
    static constexpr size_t kStatic = (P == kGradW ? 1024 : NT) * sizeof(float) + 512;
    // Operand stages, and whether all of B's chunks stay in shared memory (with two stages at least).
    static int shape(LinArgs& a, int chunks, size_t& smem) {
        for (int resident = P == kGradW ? 0 : 1; resident >= 0; --resident)
            for (int stages = kMostStages; stages >= 2; --stages) {
                smem = L::smem_bytes(stages, resident ? chunks : stages);
                if (smem > kSmemOfBlock - kStatic) continue;
                a.stages = stages;
                a.resident = resident;
                return E3J_OK;
            }
        return E3J_ERR_UNSUPPORTED;   // (never: two stages of every kind fit)
    }
    static int run(LinArgs& a, cudaStream_t st) {
        static std::atomic<uint64_t> allowed{0};
        if (int rc = allow_smem(kernel, kSmemOfBlock - kStatic, allowed)) return rc;
        const int columns = P == kGradX ? a.n_in : a.n_out, contraction = P == kGradX ? a.n_out : a.n_in;
        a.n_tiles = (columns + NT - 1) / NT;
        size_t smem = 0;
        if (int rc = shape(a, (contraction + kChunk - 1) / kChunk, smem)) return rc;
        int64_t grid;
        if (P == kGradW) {
            grid = (int64_t)a.n_tiles * a.m_tiles * a.ranges;
        } else {
            const int64_t row_tiles = (a.rows + kTileRows - 1) / kTileRows;
            const int64_t per = std::max<int64_t>(sm_count() / a.n_tiles, 1);
            grid = a.n_tiles * std::min(per, row_tiles);
            // Boxes where a block has several tiles (the map costs the host a microsecond, which small calls would wait for): 78 000 x 512
            // -> 512, no activation: 86 us by cp.async, 80 so.
            if constexpr (L::kBoxes)
                a.boxes = a.resident && row_tiles * a.n_tiles > 2 * grid &&
                          box_map(&a.map_a, P == kGradX ? a.gz : a.x, a.rows, P == kGradX ? a.ld_gz : a.n_in);
        }
        return launch_dependent(kernel, dim3((unsigned)grid), dim3(lin_threads(sizeof(T))), smem, st, a);
    }
};

// Which rows start on 16 bytes: those of A; all others (B's, and but for kGradW those of the results and of what they meet).
struct Aligned { bool a, others; };
template <Product P, class T, class G, int ACT, Chains CHAINS> int product_of(LinArgs& x, Aligned v, bool narrow, cudaStream_t st) {
    if (v.a && v.others) return narrow ? Launch<P, T, G, 64, ACT, true, true, CHAINS>::run(x, st) : Launch<P, T, G, 128, ACT, true, true, CHAINS>::run(x, st);
    if (v.a) return narrow ? Launch<P, T, G, 64, ACT, true, false, CHAINS>::run(x, st) : Launch<P, T, G, 128, ACT, true, false, CHAINS>::run(x, st);
    if (v.others) return narrow ? Launch<P, T, G, 64, ACT, false, true, CHAINS>::run(x, st) : Launch<P, T, G, 128, ACT, false, true, CHAINS>::run(x, st);
    return narrow ? Launch<P, T, G, 64, ACT, false, false, CHAINS>::run(x, st) : Launch<P, T, G, 128, ACT, false, false, CHAINS>::run(x, st);
}
template <Product P, class T, class G, int ACT = E3J_ACT_NONE> int product(LinArgs& x, Aligned v, cudaStream_t st) {
    const int columns = P == kGradX ? x.n_in : x.n_out;
    // Tiles of 64 columns instead of 128: where there are no more columns; where every one of them has an SM of its own (1218 rows of 336
    // -> 328 float32 forward: 14.9 us with tiles of 128, 11.6 so); and with float32, not in sums over rows (38 and 44 us), where they
    // leave fewer columns of the tiles empty and
    // - the rows that they meet are off 16 bytes, so that loaders and readers pay by the column (60 000 rows forward, with 128 and 64: 33 -> 161
    //   46.9 and 36.0, 97 -> 161 60.8 and 49.3, 33 -> 257 59.8 and 51.3, 33 -> 513 96.7 and 88.4, 97 -> 290 86.6 and 80.1; grad_x 161 <- 97
    //   61.2 and 54.0), or
    // - two of these hold, not in grad_x: readers have a residual or grad_y to fetch, W is one chunk, there are no more than 192 columns
    //   (all three 27.9 and 27.7; fetching, 128 -> 160 39.7 and 36.3, 256 -> 160 63.8 and 61.7, 64 -> 288 51.0 and 47.9; without, 32 -> 160 22.4
    //   and 18.8, 64 -> 192 23.8 and 22.0).
    // Not with one or none (fetching, 128 -> 288 54.7 and 57.3, 256 -> 288 87.6 and 100.0; without, 96 -> 160 27.4 and 30.5, 64 -> 288 32.3 and
    // 35.1, 128 -> 288 40.6 and 55.6; grad_x 192 <- 64 20.1 and 20.5, 288 <- 128 40.3 and 53.1).
    const int contraction = P == kGradX ? x.n_out : x.n_in;
    const int reasons = (P == kSlope || (P == kForward && x.residual)) + (contraction <= kChunk) + (columns <= 192);
    const bool fewer = P != kGradW && sizeof(T) == 4 && (columns - 1) % 128 < 64 && (!v.others || (P != kGradX && reasons >= 2));
    const bool narrow = columns <= 64 || fewer || (P != kGradW && (x.rows + kTileRows - 1) / kTileRows * ((columns + 63) / 64) <= sm_count());
    if constexpr (P != kGradW && sizeof(T) == 4) {
        if (contraction > kLongest)   // (tiles of 64: the sums of the chains are registers)
            return v.a && v.others ? Launch<P, T, G, 64, ACT, true, true, kMany>::run(x, st) : Launch<P, T, G, 64, ACT, false, false, kMany>::run(x, st);
        // (as kMany 40 000 x 512 -> 256 takes 125 us; in one chain, half as exact, 83; so 91)
        if (contraction > kChain) return product_of<P, T, G, ACT, kPair>(x, v, narrow, st);
    }
    return product_of<P, T, G, ACT, kOne>(x, v, narrow, st);
}
template <Product P, class T, class G> int product_act(LinArgs& a, int act, Aligned v, cudaStream_t st) {
    if (act == E3J_ACT_SILU) return product<P, T, G, E3J_ACT_SILU>(a, v, st);
    if (act == E3J_ACT_TANH) return product<P, T, G, E3J_ACT_TANH>(a, v, st);
    if (act == E3J_ACT_GELU) return product<P, T, G, E3J_ACT_GELU>(a, v, st);
    if constexpr (P == kForward) return product<P, T, G>(a, v, st);
    return E3J_ERR_INVALID_ARG;
}

// Rows of `ld` elements from p on start on 16 bytes and are whole 16-byte pieces (p null: so they do).
inline bool whole(const void* p, int64_t ld, size_t size) { return !p || (((uintptr_t)p | (uintptr_t)(ld * size)) & 15u) == 0; }

template <class T> int linear_fwd(LinArgs& a, int act, cudaStream_t st) {
    const Aligned v{whole(a.x, a.n_in, sizeof(T)),
                    whole(a.W, a.n_out, sizeof(T)) && whole(a.out, a.n_out, sizeof(T)) && whole(a.residual, a.n_out, sizeof(T))};
    return product_act<kForward, T, T>(a, act, v, st);
}

template <class T, class G> int gradients(LinArgs a, const BwdLayout& L, void* grad_x, void* grad_W, void* grad_b, cudaStream_t st) {
    const bool gz = whole(a.gz, a.ld_gz, sizeof(G));
    if (grad_x) {
        a.out = grad_x;
        if (int rc = product<kGradX, T, G>(a, Aligned{gz, whole(a.W, a.n_out, sizeof(T)) && whole(grad_x, a.n_in, sizeof(T))}, st)) return rc;
    }
    if (!grad_W && !grad_b) return E3J_OK;
    a.ranges = L.ranges;
    a.m_tiles = L.m_tiles;
    a.want_sums = grad_b != nullptr;
    a.beside = grad_x != nullptr;   // (1218 rows of 336 -> 328 float32, both products: 31 us one after the other, 27 so; 377 of 104 -> 140 bfloat16 32 and 18)
    a.grad_W = grad_W;
    a.grad_b = grad_b;
    if (int rc = product<kGradW, T, G>(a, Aligned{whole(a.x, a.n_in, sizeof(T)), gz}, st)) return rc;
    if (L.direct) return E3J_OK;
    return sum_shares<T>(L.ranges, (int64_t)a.n_in * a.n_out, a.n_out, a.shares, (T*)grad_W, (T*)grad_b, st);
}

template <class T, int ACT, bool VEC> int narrow_kernel(LinArgs& a, int blocks, bool direct, cudaStream_t st) {
    using S = NarrowLayout<T, ACT>;
    constexpr auto kernel = linear_bwd_narrow_kernel<T, ACT, VEC>;
    static std::atomic<uint64_t> allowed{0};
    if (int rc = allow_smem(kernel, S::smem, allowed)) return rc;
    return launch_cluster(kernel, blocks, direct ? blocks : 1, kNarrowThreads, S::smem, st, a);
}
template <class T, int ACT> int narrow_bwd(LinArgs& a, const BwdLayout& L, void* grad_W, void* grad_b, cudaStream_t st) {
    const bool vector = whole(a.x, a.n_in, sizeof(T)) && whole(a.W, a.n_out, sizeof(T)) && whole(a.grad_y, a.n_out, sizeof(T)) &&
                        whole(a.out, a.n_in, sizeof(T));
    a.grad_W = grad_W;
    a.grad_b = grad_b;
    if (int rc = vector ? narrow_kernel<T, ACT, true>(a, L.ranges, L.direct, st) : narrow_kernel<T, ACT, false>(a, L.ranges, L.direct, st)) return rc;
    if (L.direct || (!grad_W && !grad_b)) return E3J_OK;
    return sum_shares<T>(L.ranges * NarrowLayout<T, ACT>::parts, (int64_t)a.n_in * a.n_out, a.n_out, a.shares, (T*)grad_W, (T*)grad_b, st);
}

template <class T>
int linear_bwd(LinArgs& a, int act, const BwdLayout& L, void* workspace, void* grad_x, void* grad_W, void* grad_b, cudaStream_t st) {
    a.shares = L.direct ? nullptr : (float*)((char*)workspace + L.shares);
    if (L.narrow) {
        a.out = grad_x;
        if (act == E3J_ACT_SILU) return narrow_bwd<T, E3J_ACT_SILU>(a, L, grad_W, grad_b, st);
        if (act == E3J_ACT_TANH) return narrow_bwd<T, E3J_ACT_TANH>(a, L, grad_W, grad_b, st);
        if (act == E3J_ACT_GELU) return narrow_bwd<T, E3J_ACT_GELU>(a, L, grad_W, grad_b, st);
        return narrow_bwd<T, E3J_ACT_NONE>(a, L, grad_W, grad_b, st);
    }
    if (act == E3J_ACT_NONE) {
        a.gz = a.grad_y;
        a.ld_gz = a.n_out;
        return gradients<T, T>(a, L, grad_x, grad_W, grad_b, st);
    }
    a.out = workspace;
    a.ld_gz = (int)L.ld_gz;
    const Aligned v{whole(a.x, a.n_in, sizeof(T)), whole(a.W, a.n_out, sizeof(T)) && whole(a.grad_y, a.n_out, sizeof(T))};
    if (int rc = product_act<kSlope, T, float>(a, act, v, st)) return rc;
    a.gz = workspace;
    return gradients<T, float>(a, L, grad_x, grad_W, grad_b, st);
}

}  // namespace layer
}  // namespace e3j
