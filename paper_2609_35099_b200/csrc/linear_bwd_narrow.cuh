// Backward of a linear layer of up to 64 columns on both sides in one sweep (sm_100a): what a radial network's hidden layers are.
//
//   gz = grad_y act'(x W + b);  grad_x = gz W^T;  grad_W = x^T gz;  grad_b = sum_rows gz
//
// The sweep reads x and grad_y once and writes grad_x: 160 900 rows of 64 -> 64 float32 have 124 MB to move (18.9 us at the copy
// bandwidth); as three products with gz in memory it is 288 MB.  All four operands of a tile of 128 rows are images of the kind
// of linear_kernels.cuh, and each serves two products: x is the row operand of x W and, the other way round, of x^T gz; gz of gz W^T
// and of x^T gz; W stays in shared memory for both.
//
// A block is one per SM: sixteen warps work on a tile, one more issues the tensor-core instructions.  The chain of a tile is x into its
// image - x W - gz into its image - gz W^T and x^T gz - grad_x out; images are double, so the tensor cores have the next
// tile's x W and this tile's x^T gz to do while the warps read out, and the other way round.
//
// x^T gz of float32 terms: with x's images hi, mid and lo behind one another, an operand of 128 rows is 64 features of one term and the
// same 64 of the next: [hi; mid] [hi | mid] is one instruction, [hi; mid] lo and lo hi (whose second 64 rows are not
// used) are the others.  The tensor cores add with truncation (radial_gemm.cuh): after kChainTiles tiles the warps add the sums to
// totals of their own, which stay in tensor memory too, rounding.  Adding to a share in global memory instead took 22 000 cycles each time.
//
// Few rows: the blocks are one cluster, keep their shares in shared memory and add them up there; no second kernel, no workspace
// (900 rows: 10.7 us).
//
// Waits are bounded (fast::mbar_wait); no other barrier but those behind the tiles, which all threads reach, has to be met by all.
#pragma once
#include <cooperative_groups.h>

#include "linear_kernels.cuh"

namespace e3j {
namespace layer {

constexpr int kNarrow = 64;             // columns on either side
constexpr int kWorkWarps = 16;
constexpr int kNarrowThreads = kWorkWarps * 32 + 32;
constexpr int kChainTiles = 3;

template <class T, int ACT> struct NarrowLayout {
    static constexpr int x_terms = sizeof(T) == 4 ? 3 : 1;
    static constexpr int gz_terms = sizeof(T) == 4 ? 3 : ACT == E3J_ACT_NONE ? 1 : 2;   // (grad_y itself without an activation)
    static constexpr int parts = sizeof(T) == 4 ? 2 : 1;                                // shares a block: rows 0..63, 64..127 of x^T gz
    static constexpr uint32_t image = kTileRows * 128;                                  // one term of x or gz
    static constexpr uint32_t w_image = kNarrow * 128;
    // [W | x, x | gz, gz]: x^T gz may take in the panel behind x's last one
    static constexpr uint32_t off_x = x_terms * w_image, off_gz = off_x + 2 * x_terms * image;
    static constexpr size_t smem = 1024 + off_gz + 2 * (size_t)gz_terms * image;
    // tensor memory: x W, gz W^T (two accumulators each), x^T gz (up to three), totals
    static constexpr uint32_t col_z = 0, col_x = 128, col_sums = 256, col_totals = 448;
};

// which feature a column (or a permuted row) holds: the inverse of column_of
__device__ __forceinline__ int feature_of(int c) { return (c & ~15) + 4 * ((c & 7) >> 1) + ((c & 8) >> 2) + (c & 1); }

template <class T, int ACT, bool VEC>
__global__ void __launch_bounds__(kNarrowThreads, 1) linear_bwd_narrow_kernel(const __grid_constant__ LinArgs a) {
    using S = NarrowLayout<T, ACT>;
    constexpr int X = S::x_terms, G = S::gz_terms;
    constexpr bool kSlopes = ACT != E3J_ACT_NONE;   // (else x W is not needed: gz is grad_y)
    extern __shared__ unsigned char raw_smem[];
    __shared__ uint64_t x_full[2], gz_full[2], images_free[2], z_done, x_done, x_read, chain_read, drain;
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_word, drain_word;
    __shared__ __align__(16) float bias[kNarrow];
    __shared__ float sums_of_warp[kWorkWarps][16];
    unsigned char* const smem = raw_smem + ((1024u - (umma::smem_addr(raw_smem) & 1023u)) & 1023u);
    volatile int* const abort_flag = &abort_word;
    const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
    auto wait = [&](uint64_t* bar, int phase) { return fast::mbar_wait(bar, phase & 1, abort_flag, a.status); };

    if (t == 0) {
        for (int i = 0; i < 2; ++i) {
            fast::mbar_init(&x_full[i], kWorkWarps);
            fast::mbar_init(&gz_full[i], kWorkWarps);
            fast::mbar_init(&images_free[i], 1);
        }
        fast::mbar_init(&z_done, 1);
        fast::mbar_init(&x_done, 1);
        fast::mbar_init(&x_read, kWorkWarps);
        fast::mbar_init(&chain_read, kWorkWarps);
        fast::mbar_init(&drain, 1);
        abort_word = drain_word = 0;
        fast::mbar_fence_init();
    }
    fast::grid_dependency_wait();
    fast::grid_dependency_trigger();
    if (warp == kWorkWarps) umma::tmem_alloc(&tmem_slot, 512);   // (behind the wait: see linear_kernel)
    const int64_t real = real_rows(a.rows, a.n_real);
    const int64_t row_tiles = (real + kTileRows - 1) / kTileRows;
    const int tiles = (int)(row_tiles > blockIdx.x ? (row_tiles - blockIdx.x + gridDim.x - 1) / gridDim.x : 0);   // of this block
    auto row0_of = [&](int tile) { return ((int64_t)blockIdx.x + (int64_t)tile * gridDim.x) * kTileRows; };
    const bool want_x = a.out != nullptr, want_w = a.grad_W || a.grad_b;
    const int share_size = a.n_in * a.n_out + a.n_out;
    // this block's share of the parameters' gradients: in memory, or where x's images have been
    float* const share = a.shares ? a.shares + (size_t)blockIdx.x * S::parts * share_size : reinterpret_cast<float*>(smem + S::off_x);

    // x with its columns, W with its rows and columns in column_of's order
    using OpX = Operand<T, X, kTileRows, kNarrow, true, VEC, kWorkWarps * 32>;
    OpX op_x;
    auto load_x = [&](int tile) { op_x.load(t, (const T*)a.x, a.n_in, row0_of(tile), real, 0, a.n_in); };
    if (warp < kWorkWarps && tiles > 0) load_x(0);
    if (t < 256) {
        Operand<T, X, kNarrow, kNarrow, true, VEC, 256> op_w;
        op_w.load(t, (const T*)a.W, a.n_out, 0, a.n_in, 0, a.n_out);
        op_w.template store<true>(t, smem);
        umma::fence_smem_to_async();
    } else if (t < 256 + kNarrow) {
        bias[t - 256] = a.b && t - 256 < a.n_out ? to_float(((const T*)a.b)[t - 256]) : 0.f;
    }
    umma::fence_before_sync();
    __syncthreads();
    umma::fence_after_sync();
    const uint32_t tmem = tmem_slot;
    float2 sum_b[2] = {both(0.f), both(0.f)};   // of this lane's four features

    if (warp == kWorkWarps) {
        // ------------------------------------------------ tensor cores
        if (lane == 0 && tiles > 0) {
            const uint32_t aw = umma::smem_addr(smem);
            auto image_x = [&](int tile) { return aw + S::off_x + (tile & 1) * X * S::image; };
            auto image_gz = [&](int tile) { return aw + S::off_gz + (tile & 1) * G * S::image; };
            // D0 = A_hi B_hi, D1 = the other terms; k-steps of 16
            auto products = [&](uint32_t d, uint32_t pa, uint32_t b_leading, uint32_t b_step, bool b_mn, int steps, int terms_a) {
                const uint32_t one = idesc_bf16(kTileRows, kNarrow, false, b_mn), two = idesc_bf16(kTileRows, 2 * kNarrow, false, b_mn);
                for (int k = 0; k < steps; ++k) {
                    auto da = [&](int term) { return swizzled_desc(pa + term * S::image + k * 32, 0, 1024); };
                    auto db = [&](int term) { return swizzled_desc(aw + term * S::w_image + k * b_step, b_leading, 1024); };
                    if constexpr (X == 3) {
                        mma_bf16(d, da(0), db(0), two, k > 0);
                        mma_bf16(d + kNarrow, da(1), db(0), one, 1);
                        mma_bf16(d + kNarrow, da(1), db(1), one, 1);
                        mma_bf16(d + kNarrow, da(0), db(2), one, 1);
                        mma_bf16(d + kNarrow, da(2), db(0), one, 1);
                    } else {
                        mma_bf16(d, da(0), db(0), one, k > 0);
                        if (terms_a == 2) mma_bf16(d, da(1), db(0), one, 1);
                    }
                }
            };
            auto x_times_w = [&](int tile) {
                if (!wait(&x_full[tile & 1], tile >> 1)) return false;
                umma::fence_after_sync();
                if constexpr (kSlopes) {
                    products(tmem + S::col_z, image_x(tile), S::w_image, 2048, true, (a.n_in + 15) / 16, X);
                    umma::commit(&z_done);
                }
                return true;
            };
            bool ok = x_times_w(0);
            for (int tile = 0; ok && tile < tiles; ++tile) {
                if (!(ok = wait(&gz_full[tile & 1], tile >> 1))) break;
                if (want_x) {
                    if (tile > 0 && !(ok = wait(&x_read, tile - 1))) break;
                    umma::fence_after_sync();
                    products(tmem + S::col_x, image_gz(tile), 0, 32, false, (a.n_out + 15) / 16, G);
                    umma::commit(&x_done);
                }
                if (tile + 1 < tiles && !(ok = x_times_w(tile + 1))) break;
                if (want_w) {
                    const int place = tile % kChainTiles;   // in the chain
                    if (tile > 0 && place == 0 && !(ok = wait(&chain_read, tile / kChainTiles - 1))) break;
                    umma::fence_after_sync();
                    constexpr uint32_t one = idesc_bf16(kTileRows, kNarrow, true, true);
                    constexpr uint32_t two = idesc_bf16(kTileRows, (G > 1 ? 2 : 1) * kNarrow, true, true);
                    const uint32_t d = tmem + S::col_sums, ax = image_x(tile), ag = image_gz(tile);
                    for (int k = 0; k < kTileRows / 16; ++k) {
                        const uint32_t add = k > 0 || place > 0;
                        auto dx = [&](int term) { return swizzled_desc(ax + term * S::image + k * 2048, S::image, 1024); };
                        auto dg = [&](int term) { return swizzled_desc(ag + term * S::image + k * 2048, S::image, 1024); };
                        mma_bf16(d, dx(0), dg(0), two, add);                        // [hi; mid] [hi | mid]
                        if constexpr (X == 3) {
                            mma_bf16(d + kNarrow, dx(0), dg(2), one, 1);            // [hi; mid] lo
                            mma_bf16(d + 2 * kNarrow, dx(2), dg(0), one, add);      // [lo; -] hi
                        }
                    }
                }
                umma::commit(&images_free[tile & 1]);
            }
            // everything issued is over before tensor memory goes back, also after a wait that ran out
            umma::commit(&drain);
            fast::mbar_wait(&drain, 0, &drain_word, a.status);
        }
        __syncwarp();
    } else {
        // ------------------------------------------------ the tiles' work: 32 rows and 16 columns a warp
        const int quarter = warp & 3, col = (warp >> 2) * 16;
        const int f = col + 4 * (lane & 3);           // this lane's four features
        const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)col;
        unsigned char* const x_images = smem + S::off_x;
        unsigned char* const gz_images = smem + S::off_gz;
        Quad<T> g_raw[2][2];
        auto load_g = [&](int tile) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int64_t row = row0_of(tile) + quarter * 32 + r * 8 + lane / 4;
                load_quad<VEC>(g_raw[r >> 1][r & 1], (const T*)a.grad_y + row * a.n_out + f, row < real ? a.n_out - f : 0);
            }
        };
        auto hand_over = [&](uint64_t* bar) {         // this warp's part of an image, to the tensor cores
            umma::fence_smem_to_async();
            umma::fence_before_sync();
            __syncwarp();
            if (lane == 0) fast::mbar_arrive(bar);
        };
        auto read = [&](uint32_t column, int h, Quads& v) {
            const uint32_t taddr = lanes + ((uint32_t)(h * 16) << 16) + column;
            __syncwarp();
            tmem_ld_quads(taddr, v);
            if constexpr (X == 3) {
                Quads u;
                tmem_ld_quads(taddr + kNarrow, u);
                umma::tmem_ld_wait();
                add_quads(v, u);
            } else {
                umma::tmem_ld_wait();
            }
        };
        // x^T gz of the chain that ends with `tile` -> totals, or (the last) totals and it -> this block's shares
        auto end_chain = [&](int tile) {
            if (!wait(&images_free[tile & 1], tile >> 1)) return;
            umma::fence_after_sync();
            const bool more = tile >= kChainTiles, last = tile == tiles - 1;
            const int part = quarter >> 1;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t taddr = lanes + ((uint32_t)(h * 16) << 16);
                Quads v, u, w;
                __syncwarp();
                tmem_ld_quads(taddr + S::col_sums, v);
                if constexpr (G > 1) tmem_ld_quads(taddr + S::col_sums + kNarrow, u);
                if constexpr (X == 3) tmem_ld_quads(taddr + S::col_sums + 2 * kNarrow, w);   // (rows 64 .. 127 of it are nothing)
                umma::tmem_ld_wait();
                if constexpr (X == 3)
                    if (part == 0) add_quads(u, w);
                if constexpr (G > 1) add_quads(v, u);
                if (more) {
                    tmem_ld_quads(taddr + S::col_totals, u);
                    umma::tmem_ld_wait();
                    add_quads(v, u);
                }
                if (!last) {
                    tmem_st_quads(taddr + S::col_totals, v);
                    umma::tmem_st_wait();
                } else if (part < S::parts) {
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        const int k = feature_of((quarter & 1) * 32 + h * 16 + s * 8 + lane / 4);
                        if (k < a.n_in) store_quad<false>(share + part * share_size + k * a.n_out + f, v.p[s], a.n_out - f);
                    }
                }
            }
            umma::fence_before_sync();
            __syncwarp();
            if (lane == 0) fast::mbar_arrive(&chain_read);
        };

        if (tiles > 0) {
            op_x.store(t, x_images);
            hand_over(&x_full[0]);
            load_g(0);
            if (tiles > 1) load_x(1);
        }
        for (int tile = 0; tile < tiles; ++tile) {
            if constexpr (kSlopes) {
                if (!wait(&z_done, tile)) break;
                umma::fence_after_sync();
            }
            // (this gz image was last used with the x image that tile - 1 has waited for)
            unsigned char* const image = gz_images + (size_t)(tile & 1) * G * S::image;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                Quads v;
                if constexpr (kSlopes) read(S::col_z, h, v);
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    float2 g[2] = {both(0.f), both(0.f)};
                    g_raw[h][s].add_to(g);
                    if constexpr (kSlopes) {
                        const float4 b = *reinterpret_cast<const float4*>(bias + f);
                        const float2 z[2] = {__fadd2_rn(v.p[s][0], make_float2(b.x, b.y)), __fadd2_rn(v.p[s][1], make_float2(b.z, b.w))};
                        times_slope_as<ACT, T>(g, z);
                    }
                    sum_b[0] = __fadd2_rn(sum_b[0], g[0]);
                    sum_b[1] = __fadd2_rn(sum_b[1], g[1]);
                    // columns 2 q, 2 q + 1 of the first and of the second piece of this group of 16
                    const int row = quarter * 32 + h * 16 + s * 8 + lane / 4;
                    unsigned char* const at = image + image_offset(row, col / 8) + (lane & 3) * 4;
                    unsigned char* const behind = image + image_offset(row, col / 8 + 1) + (lane & 3) * 4;
                    uint2 terms[G];
                    split<G>(g[0], g[1], terms);
#pragma unroll
                    for (int k = 0; k < G; ++k) {
                        *reinterpret_cast<uint32_t*>(at + k * S::image) = terms[k].x;
                        *reinterpret_cast<uint32_t*>(behind + k * S::image) = terms[k].y;
                    }
                }
            }
            hand_over(&gz_full[tile & 1]);
            if (tile + 1 < tiles) {
                if (tile > 0 && !wait(&images_free[(tile + 1) & 1], (tile - 1) >> 1)) break;
                op_x.store(t, x_images + (size_t)((tile + 1) & 1) * X * S::image);
                hand_over(&x_full[(tile + 1) & 1]);
                load_g(tile + 1);
                if (tile + 2 < tiles) load_x(tile + 2);
            }
            if (want_w && tile > 0 && tile % kChainTiles == 0) end_chain(tile - 1);
            if (want_x) {
                if (!wait(&x_done, tile)) break;
                umma::fence_after_sync();
                if (col < a.n_in) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        Quads v;
                        read(S::col_x, h, v);
#pragma unroll
                        for (int s = 0; s < 2; ++s) {
                            const int64_t row = row0_of(tile) + quarter * 32 + h * 16 + s * 8 + lane / 4;
                            if (row < real) store_quad<VEC>((T*)a.out + row * a.n_in + f, v.p[s], a.n_in - f);
                        }
                    }
                }
                umma::fence_before_sync();
                __syncwarp();
                if (lane == 0) fast::mbar_arrive(&x_read);
            }
        }
        if (want_w) {
            if (tiles > 0) end_chain(tiles - 1);
            else
                for (int i = t; i < S::parts * share_size; i += kWorkWarps * 32) share[i] = 0.f;
            // the column sums: over the warp's rows, then over the four warps of a column group in order
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float v = i & 1 ? sum_b[i / 2].y : sum_b[i / 2].x;
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) v += __shfl_xor_sync(~0u, v, o);
                if (lane < 4) sums_of_warp[warp][4 * lane + i] = v;
            }
        }
        if (want_x && real < a.rows) {
            T* const out = (T*)a.out;
            for (int64_t i = real * a.n_in + blockIdx.x * (int64_t)(kWorkWarps * 32) + t; i < a.rows * a.n_in; i += (int64_t)gridDim.x * (kWorkWarps * 32))
                out[i] = from_float<T>(0.f);
        }
    }
    umma::fence_before_sync();
    __syncthreads();
    umma::fence_after_sync();
    // Tensor memory goes back before the cluster's blocks wait for one another: a block that has not got its own yet may be waiting for
    // that of a block of another cluster, whose peer waits for this cluster's.
    if (warp == kWorkWarps) umma::tmem_dealloc(tmem, 512);
    if (want_w && t < a.n_out) {
        float sum = 0.f;
        for (int q = 0; q < 4; ++q) sum += sums_of_warp[(t >> 4) * 4 + q][t & 15];
        share[share_size - a.n_out + t] = sum;
        if (S::parts == 2) share[2 * share_size - a.n_out + t] = 0.f;
    }
    if (want_w && !a.shares) {   // the shares of the cluster's blocks, added in their order
        const auto cluster = cooperative_groups::this_cluster();
        cluster.sync();
        for (int i = blockIdx.x * kNarrowThreads + t; i < share_size; i += gridDim.x * kNarrowThreads) {
            float theirs[kClusterBlocks][S::parts], sum = 0.f;   // (all on their way before the first is added)
#pragma unroll
            for (int r = 0; r < kClusterBlocks; ++r)
#pragma unroll
                for (int p = 0; p < S::parts; ++p) theirs[r][p] = r < (int)gridDim.x ? cluster.map_shared_rank(share, r)[p * share_size + i] : 0.f;
#pragma unroll
            for (int r = 0; r < kClusterBlocks; ++r)
#pragma unroll
                for (int p = 0; p < S::parts; ++p) sum += theirs[r][p];
            const int in_W = share_size - a.n_out;
            if (i < in_W && a.grad_W) ((T*)a.grad_W)[i] = from_float<T>(sum);
            if (i >= in_W && a.grad_b) ((T*)a.grad_b)[i - in_W] = from_float<T>(sum);
        }
        cluster.sync();   // (nobody leaves while others read)
    }
}

}  // namespace layer
}  // namespace e3j
