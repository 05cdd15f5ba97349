// Products of the linear layer on the fifth-generation tensor cores (sm_100a): forward, and the three products of its
// backward, for float32 and bfloat16.
//
// Operands.  The tensor cores multiply bfloat16 pairs into float32 accumulators (tcgen05.mma kind::f16).  A float32 value is the
// exact sum of three bfloat16 (24 significant bits are three times 8): v = hi + mid + lo, each the leading bits of what
// is left, cut off and subtracted.  A product of two float32 is the sum of the six term products of weight 2^-16 and more; the
// three left out are below 2^-22 of it.  That is as many tensor-core passes as the three-product TF32 form (whose products run at
// half the rate), from 6 bytes of shared memory an element instead of 8, and with operands of 16 bits that the tensor cores take
// along either dimension: x is the row operand of x W and the column operand of x^T gz from the same kind of image, with no
// transposed copy of anything.  The float32 gradient gz of a bfloat16 layer is split into two terms (16 bits, the second rounded
// to nearest), so it reaches both products of the backward without the loss of a rounding to bfloat16; bfloat16 tensors are one term.
//
// Image of a matrix block in shared memory: panels of 64 columns, 128 bytes a row, 16-byte pieces at (piece ^ row % 8): the 128-byte
// swizzle.  With the panel's rows as the operand's rows it is K-major, with them as the contraction it is MN-major;
// which, the instruction descriptor says.
//
// Accumulators.  The tensor cores add with truncation, so long chains drift (see radial_gemm.cuh).  Of float32 operands the
// hi hi products go to one accumulator and the five smaller ones to another (B's hi and mid lie behind one another, so the first
// two are one instruction of twice the width), and a chain ends after kChain of the contraction, 16 additions of hi hi: the readers
// add the chains, rounding: in products over up to kLongest columns when they read a tile, whose two chains are in accumulator
// sets of their own (PAIR); beyond that, and over rows, in registers (LONG).
// An instruction of 16 products loses 3 half steps of the sum on average (measured: each product is cut off at a quarter of a half
// step of the sum, and the sum at a whole step).  2-norm of the error, normal values: 1.1e-7 with 64 columns, 2.8e-7 with 256, 512
// (5.3e-7 in one chain) and 4096 (4.6e-6).
//
// Order of a tile's columns.  A quad of lanes reads tensor memory in pieces of 8 columns, two a lane (tcgen05.ld 16x256b).  Columns
// of a 16-column group are dealt out so that the two pieces of a lane are four consecutive features: rows leave in 64-byte (float32) or
// 32-byte (bfloat16) runs a quad, whole sectors, without a detour through shared memory.  (column_of)
//
// A block is one per SM and has three roles: eight warps fetch, split and store operands (one chunk in registers ahead; bfloat16 rows
// that start on 16 bytes go to shared memory by cp.async, up to four chunks ahead, or in large calls as boxes of a tensor map, which one
// thread asks for, as many ahead as there are stages), one issues the tensor-core instructions, eight
// (bfloat16: sixteen) read accumulators and finish tiles.  Operand stages and accumulator sets stand between them.  As one role of 256 threads
// that took turns, two blocks an SM, 160 900 x 64 -> 64 float32 took 25.7 us instead of 22.4.  Waits are bounded (fast::mbar_wait).
#pragma once
#include "layer_common.cuh"
#include "linear.hpp"
#include "umma.cuh"

namespace e3j {
namespace layer {

constexpr int kRoleThreads = 256;   // loaders
// Reading warps: sixteen, but for float32, whose loaders need the registers, eight (60 000 x 256 -> 256 with residual, with sixteen: 122 us).
constexpr int read_warps(int size) { return size == 4 ? 8 : 16; }
constexpr int lin_threads(int size) { return read_warps(size) * 32 + kRoleThreads + 32; }
constexpr int kMostStages = 6;
constexpr int kTileRows = 128;      // accumulator lanes
constexpr int kChunk = 64;          // contraction elements a chunk
constexpr int kChain = 256;         // contraction elements a chain is long (float32)
constexpr int kLongest = 2 * kChain;   // ... up to which the two accumulator sets hold a tile's chains

// ---------------------------------------------------------------- operands
// Four consecutive elements, `left` of which are there, as they lie in memory.
template <class T> struct Quad;
template <> struct Quad<float> {
    float4 q;
    __device__ __forceinline__ void add_to(float2 (&v)[2]) const {
        v[0] = __fadd2_rn(v[0], make_float2(q.x, q.y));
        v[1] = __fadd2_rn(v[1], make_float2(q.z, q.w));
    }
};
template <> struct Quad<bf16> {
    uint2 q;
    __device__ __forceinline__ void add_to(float2 (&v)[2]) const {
        v[0] = __fadd2_rn(v[0], make_float2(low_float(q.x), high_float(q.x)));
        v[1] = __fadd2_rn(v[1], make_float2(low_float(q.y), high_float(q.y)));
    }
};
template <bool VEC> __device__ __forceinline__ void load_quad(Quad<float>& v, const float* from, int left) {
    v.q = make_float4(0.f, 0.f, 0.f, 0.f);
    if constexpr (VEC) {
        if (left >= 4) v.q = __ldg(reinterpret_cast<const float4*>(from));
    } else {
        // (four predicates, no branch: the loads of all quads go out together)
        if (left > 0) v.q.x = __ldg(from);
        if (left > 1) v.q.y = __ldg(from + 1);
        if (left > 2) v.q.z = __ldg(from + 2);
        if (left > 3) v.q.w = __ldg(from + 3);
    }
}
template <bool VEC> __device__ __forceinline__ void load_quad(Quad<bf16>& v, const bf16* from, int left) {
    v.q = make_uint2(0, 0);
    if constexpr (VEC) {
        if (left >= 4) v.q = __ldg(reinterpret_cast<const uint2*>(from));
    } else {
        const uint16_t* const h = reinterpret_cast<const uint16_t*>(from);
        if (left > 0) v.q.x = __ldg(h);
        if (left > 1) v.q.x |= (uint32_t)__ldg(h + 1) << 16;
        if (left > 2) v.q.y = __ldg(h + 2);
        if (left > 3) v.q.y |= (uint32_t)__ldg(h + 3) << 16;
    }
}
template <bool VEC, class T> __device__ __forceinline__ void store_quad(T* to, const float2 (&v)[2], int left) {
    if constexpr (VEC) {
        if (left >= 4) store_four(to, v);
    } else {
        if (left > 0) to[0] = from_float<T>(v[0].x);
        if (left > 1) to[1] = from_float<T>(v[0].y);
        if (left > 2) to[2] = from_float<T>(v[1].x);
        if (left > 3) to[3] = from_float<T>(v[1].y);
    }
}

// Cuts the leading 8 bits off two values: a term of both, packed; what is left of them in v.
__device__ __forceinline__ uint32_t cut_pair(float2& v) {
    const uint32_t p = __byte_perm(__float_as_uint(v.x), __float_as_uint(v.y), 0x7632);
    v = __fadd2_rn(v, make_float2(-low_float(p), -high_float(p)));
    return p;
}
// The terms of four elements, packed in pairs; the last is rounded (of three it is exact).
template <int TERMS> __device__ __forceinline__ void split(float2 a, float2 b, uint2 (&t)[TERMS]) {
#pragma unroll
    for (int k = 0; k + 1 < TERMS; ++k) t[k] = make_uint2(cut_pair(a), cut_pair(b));
    t[TERMS - 1] = make_uint2(pack_bf16(a.x, a.y), pack_bf16(b.x, b.y));
}
template <int TERMS> __device__ __forceinline__ void split(const Quad<float>& v, uint2 (&t)[TERMS]) {
    split<TERMS>(make_float2(v.q.x, v.q.y), make_float2(v.q.z, v.q.w), t);
}
template <int TERMS> __device__ __forceinline__ void split(const Quad<bf16>& v, uint2 (&t)[TERMS]) {
    static_assert(TERMS == 1, "bfloat16 is one term");
    t[0] = v.q;
}

__device__ __forceinline__ uint32_t image_offset(int row, int piece) { return (uint32_t)(row * 128 + ((piece ^ (row & 7)) << 4)); }
// where a feature of a 16-feature group lies among the tile's columns
__device__ __forceinline__ int column_of(int f) { return 2 * ((f & 15) >> 2) + (f & 1) + ((f & 2) << 2) + (f & ~15); }

// Matrix descriptor: 128-byte swizzle.  K-major: `stride` between groups of 8 rows (the other offset is not used).  MN-major:
// `stride` between groups of 8 of the contraction, `leading` between panels.
__device__ __forceinline__ uint64_t swizzled_desc(uint32_t address, uint32_t leading, uint32_t stride) {
    const uint32_t lo = ((address >> 4) & 0x3FFFu) | (((leading >> 4) & 0x3FFFu) << 16);
    const uint32_t hi = ((stride >> 4) & 0x3FFFu) | (1u << 14) | (2u << 29);
    return ((uint64_t)hi << 32) | lo;
}
__host__ __device__ constexpr uint32_t idesc_bf16(int m, int n, bool a_mn, bool b_mn) {
    return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) | ((uint32_t)(n >> 3) << 17) |
           ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ void mma_bf16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// 16 lanes x 16 columns of tensor memory: p[s] are four consecutive features (column_of) of row lane / 4 + 8 s; a quad of lanes has the
// group's 16.  Columns 2 (lane % 4) and the next one, of the first and of the second 8.
struct Quads { float2 p[2][2]; };
__device__ __forceinline__ void tmem_ld_quads(uint32_t taddr, Quads& v) {
    uint32_t r[8];
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(taddr) : "memory");
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 0; i < 2; ++i) v.p[s][i] = make_float2(__uint_as_float(r[4 * i + 2 * s]), __uint_as_float(r[4 * i + 2 * s + 1]));
}
__device__ __forceinline__ void tmem_st_quads(uint32_t taddr, const Quads& v) {
    asm volatile("tcgen05.st.sync.aligned.16x256b.x2.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 ::"r"(taddr), "r"(__float_as_uint(v.p[0][0].x)), "r"(__float_as_uint(v.p[0][0].y)), "r"(__float_as_uint(v.p[1][0].x)),
                   "r"(__float_as_uint(v.p[1][0].y)), "r"(__float_as_uint(v.p[0][1].x)), "r"(__float_as_uint(v.p[0][1].y)),
                   "r"(__float_as_uint(v.p[1][1].x)), "r"(__float_as_uint(v.p[1][1].y)) : "memory");
}
__device__ __forceinline__ void add_quads(Quads& v, const Quads& u) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v.p[i >> 1][i & 1] = __fadd2_rn(v.p[i >> 1][i & 1], u.p[i >> 1][i & 1]);
}

// Operand block of ROWS rows and COLS columns, fetched in quads (a warp's accesses are contiguous: 16 or 32 lanes a row), its columns
// in order or in column_of's (PERMUTED).  Shared memory is written without bank conflicts either way.
template <class T, int TERMS, int ROWS, int COLS, bool PERMUTED, bool VEC, int THREADS = kRoleThreads> struct Operand {
    static constexpr int kAcross = COLS / 4, kRows = THREADS / kAcross;   // quads a row, rows a pass
    static constexpr int kItems = ROWS / kRows;
    static constexpr uint32_t kTermBytes = ROWS * COLS * 2;
    static constexpr uint32_t kBytes = TERMS * kTermBytes;
    static_assert(THREADS % kAcross == 0 && ROWS % kRows == 0 && kRows % 8 == 0, "whole passes, and a thread's rows at one place of the swizzle");
    Quad<T> q[kItems];

    // rows [row0, row_end) and columns [col0, col_end) of `from` are there, the rest is zero; t: this thread
    __device__ __forceinline__ void load(int t, const T* from, int64_t ld, int64_t row0, int64_t row_end, int col0, int col_end) {
        const int row = t / kAcross, col = col0 + t % kAcross * 4;
        const int rows = (int)min(row_end - row0, (int64_t)ROWS);
        const T* at = from + (row0 + row) * ld + col;
        const int64_t step = ld * kRows;
#pragma unroll
        for (int i = 0; i < kItems; ++i, at += step) load_quad<VEC>(q[i], at, row + i * kRows < rows ? col_end - col : 0);
    }
    // PERMUTE_ROWS: the block's rows become the tile's columns
    template <bool PERMUTE_ROWS = false>
    __device__ __forceinline__ void store(int t, unsigned char* image) const {
        static_assert(!PERMUTE_ROWS || kRows % 16 == 0, "a thread's rows at one place of their groups of 16");
        const int across = t % kAcross, row = PERMUTE_ROWS ? column_of(t / kAcross) : t / kAcross;
        unsigned char* const panel = image + (across >> 4) * (ROWS * 128);
        const uint32_t at = PERMUTED ? image_offset(row, (across >> 1) & 6) + (across & 3) * 4
                                     : image_offset(row, (across >> 1) & 7) + (across & 1) * 8;
        const uint32_t behind = image_offset(row, ((across >> 1) & 6) + 1) + (across & 3) * 4;
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            uint2 t2[TERMS];
            split<TERMS>(q[i], t2);
#pragma unroll
            for (int k = 0; k < TERMS; ++k) {
                unsigned char* const to = panel + i * (kRows * 128) + k * kTermBytes;
                if constexpr (PERMUTED) {
                    *reinterpret_cast<uint32_t*>(to + at) = t2[k].x;
                    *reinterpret_cast<uint32_t*>(to + behind) = t2[k].y;
                } else {
                    *reinterpret_cast<uint2*>(to + at) = t2[k];
                }
            }
        }
    }
};

// The same block straight into shared memory (one term, rows that start on 16 bytes): 16-byte pieces, zeros where nothing is.
template <int ROWS, int COLS>
__device__ __forceinline__ void copy_async(int t, uint32_t image, const bf16* from, int64_t ld, int64_t row0, int64_t row_end,
                                           int col0, int col_end) {
    constexpr int kAcross = COLS / 8, kItems = ROWS * kAcross / kRoleThreads, kRows = kRoleThreads / kAcross;
    const int row = t / kAcross, across = t % kAcross, col = col0 + across * 8;
    const int rows = col < col_end ? (int)min(row_end - row0, (int64_t)ROWS) : 0;
    const bf16* at = from + (row0 + row) * ld + col;
    const int64_t step = ld * kRows;
    static_assert(kRows % 8 == 0, "an item's place in the swizzle is the same for all items");
    const uint32_t to = image + (across >> 3) * (ROWS * 128) + image_offset(row, across & 7);
#pragma unroll
    for (int i = 0; i < kItems; ++i, at += step) {
        const bool there = row + i * kRows < rows;
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + i * kRows * 128), "l"(there ? at : from),
                     "r"(there ? 16 : 0) : "memory");
    }
}
// A box of a tensor map with the 128-byte swizzle into an image; x a multiple of 8 columns.
__device__ __forceinline__ void load_box(uint32_t image, const CUtensorMap* map, int x, int y, uint64_t* bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(image), "l"(map), "r"(x), "r"(y), "r"(fast::smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// all but the newest `n` groups have arrived
__device__ __forceinline__ void async_wait(int n) {
    if (n >= 3) asm volatile("cp.async.wait_group 3;" ::: "memory");
    else if (n == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
    else if (n == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
    else asm volatile("cp.async.wait_group 0;" ::: "memory");
}

// ---------------------------------------------------------------- the kernel
// T: type of the layer's tensors; G: type of gz (kGradX, kGradW).
template <Product P, class T, class G> struct Types {
    using A = T; using B = T;
    static constexpr int a_terms = sizeof(T) == 4 ? 3 : 1, b_terms = a_terms;
};
template <class T, class G> struct Types<kGradX, T, G> {
    using A = G; using B = T;
    static constexpr int b_terms = sizeof(T) == 4 ? 3 : 1, a_terms = sizeof(G) == 2 ? 1 : sizeof(T) == 4 ? 3 : 2;
};
template <class T, class G> struct Types<kGradW, T, G> {
    using A = T; using B = G;
    static constexpr int a_terms = sizeof(T) == 4 ? 3 : 1, b_terms = sizeof(G) == 2 ? 1 : sizeof(T) == 4 ? 3 : 2;
};

// VA: A's rows start on 16 bytes; VO: those of B, of the results and of what they meet do.
// CHAINS of float32 products that a tile's contraction is cut into: kOne; kPair, one in either of two accumulator sets (more than kChain
// columns); kMany, added in registers (more than kLongest).
enum Chains { kOne, kPair, kMany };
template <Product P, class T, class G, int NT, bool VA, bool VO, Chains CHAINS> struct LinTile {
    using Ty = Types<P, T, G>;
    static constexpr bool kRowSum = P == kGradW;    // contraction over rows: both operands MN-major
    // Sums over rows of float32 take 32 rows at a time: with 64 the loaders' registers do not hold both operands of a chunk, and what
    // is spilled is waited for (backward of 60 000 x 128 -> 128: 81 us against 77).
    static constexpr int kRows = kRowSum && Ty::a_terms == 3 ? 32 : kChunk;
    using OpA = Operand<typename Ty::A, Ty::a_terms, kRowSum ? kRows : kTileRows, kRowSum ? kTileRows : kChunk, false, VA>;
    using OpB = Operand<typename Ty::B, Ty::b_terms, P == kGradX ? NT : kRows, P == kGradX ? kChunk : NT, P != kGradX, VO>;
    static constexpr bool kA_mn = kRowSum, kB_mn = P != kGradX;
    static constexpr int kSets = Ty::a_terms == 3 ? 2 : 1;     // accumulators of a chain
    static constexpr int kUnits = CHAINS == kPair && NT == 64 ? 4 : 2;   // chains in tensor memory: two tiles' (kPair with NT 128: one's)
    static constexpr int kColumns = kUnits * kSets * NT;
    static constexpr bool kAsyncA = VA && sizeof(typename Ty::A) == 2;   // A by cp.async ...
    static constexpr bool kBoxes = kAsyncA && !kRowSum;                  // ... or by tiled bulk copies (LinArgs::boxes)
    static size_t smem_bytes(int stages, int b_slots) { return 1024 + (size_t)stages * OpA::kBytes + (size_t)b_slots * OpB::kBytes; }
};

template <Product P, class T, class G, int NT, int ACT, bool VA, bool VO, Chains CHAINS>
__global__ void __launch_bounds__(lin_threads(sizeof(T)), 1) linear_kernel(const __grid_constant__ LinArgs a) {
    using L = LinTile<P, T, G, NT, VA, VO, CHAINS>;
    using TA = typename L::Ty::A;
    using TB = typename L::Ty::B;
    using OpA = typename L::OpA;
    using OpB = typename L::OpB;
    constexpr int kTermsA = L::Ty::a_terms, kTermsB = L::Ty::b_terms;
    constexpr bool LONG = CHAINS == kMany, PAIR = CHAINS == kPair;
    static_assert(!PAIR || (P != kGradW && L::kSets == 2), "two accumulators a chain, a chain in either set");
    constexpr int kChunkRows = L::kRows, kGroupChunks = kChain / L::kRows;   // chunks a chain
    extern __shared__ unsigned char raw_smem[];
    __shared__ uint64_t full[kMostStages], empty[kMostStages], tile_full[4], tile_empty[4], drain;
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_word, drain_word;
    __shared__ float column_sums[P == kGradW ? OpB::kRows * NT : 1];   // (1024)
    __shared__ __align__(16) float bias[P == kForward || P == kSlope ? NT : 4];
    unsigned char* const smem = raw_smem + ((1024u - (umma::smem_addr(raw_smem) & 1023u)) & 1023u);
    volatile int* const abort_flag = &abort_word;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    constexpr int kLoaders = kRoleThreads / 32, kReaders = read_warps(sizeof(T)), kIssuer = kReaders + kLoaders;
    constexpr int kWarpColumns = NT / (kReaders / 4);   // of a reading warp

    if (threadIdx.x == 0) {
        for (int i = 0; i < kMostStages; ++i) { fast::mbar_init(&full[i], L::kBoxes && a.boxes ? 1 : kLoaders); fast::mbar_init(&empty[i], 1); }
        for (int i = 0; i < L::kUnits; ++i) { fast::mbar_init(&tile_full[i], 1); fast::mbar_init(&tile_empty[i], kReaders); }
        fast::mbar_init(&drain, 1);
        abort_word = drain_word = 0;
        fast::mbar_fence_init();
    }
    // Sums over rows that follow grad_x's product do not need it: they run beside it, and their wait for it comes at their end (the second
    // exception of fast::grid_dependency_wait).  They start when every block of that product has got as far as its trigger, behind its
    // wait; so gz, x and the rest are written.  That these writes are seen is not that wait's promise to this kernel: a fence
    // before the product's trigger and one here hand on what the product's threads may see.
    const bool beside = P == kGradW && a.beside;
    if (beside) __threadfence();
    else fast::grid_dependency_wait();
    if (P == kGradX) __threadfence();
    fast::grid_dependency_trigger();
    // (a block that waits for another kernel holds no tensor memory, which a block of that kernel may be waiting for)
    if (warp == kIssuer) umma::tmem_alloc(&tmem_slot, L::kColumns);
    const int nt = blockIdx.x % a.n_tiles;
    const int n0 = nt * NT;
    if constexpr (P == kForward || P == kSlope)
        if (threadIdx.x < NT)
            bias[threadIdx.x] = a.b && n0 + (int)threadIdx.x < a.n_out ? to_float(((const T*)a.b)[n0 + threadIdx.x]) : 0.f;
    const int64_t real = real_rows(a.rows, a.n_real);

    // ---- what this block does: units (a tile, or for kGradW, LONG and PAIR a chain of one tile) of up to `chunks` chunks
    int units, chunks, m0 = 0;
    int chains = 1;                            // LONG: units of a tile (PAIR: two)
    int64_t unit0 = 0, unit_step = 1;          // row tiles of this block
    int64_t chunk_begin = 0, chunk_end = 0;    // kGradW: chunks of rows of this block
    if constexpr (P == kGradW) {
        const int tile = blockIdx.x % (a.n_tiles * a.m_tiles), range = blockIdx.x / (a.n_tiles * a.m_tiles);
        m0 = tile / a.n_tiles * kTileRows;
        const int64_t all = (real + kChunkRows - 1) / kChunkRows;
        chunk_begin = all * range / a.ranges;
        chunk_end = all * (range + 1) / a.ranges;
        units = (int)((chunk_end - chunk_begin + kGroupChunks - 1) / kGroupChunks);
        chunks = kGroupChunks;
    } else {
        const int64_t tiles = (real + kTileRows - 1) / kTileRows;
        unit0 = blockIdx.x / a.n_tiles;
        unit_step = gridDim.x / a.n_tiles;
        units = (int)(tiles > unit0 ? (tiles - unit0 + unit_step - 1) / unit_step : 0);
        chunks = ((P == kGradX ? a.n_out : a.n_in) + kChunk - 1) / kChunk;
        if constexpr (LONG) {
            chains = (chunks + kGroupChunks - 1) / kGroupChunks;
            units *= chains;
        }
        if constexpr (PAIR) units *= 2;
    }
    // of a unit: its tile's first row, its first chunk
    auto row_of = [&](int unit) { return (unit0 + (LONG ? unit / chains : PAIR ? unit >> 1 : unit) * unit_step) * kTileRows; };
    auto first_chunk = [&](int unit) { return LONG ? unit % chains * kGroupChunks : PAIR ? (unit & 1) * kGroupChunks : 0; };
    auto chunks_of = [&](int unit) {
        if constexpr (P == kGradW) return (int)min((int64_t)kGroupChunks, chunk_end - chunk_begin - (int64_t)unit * kGroupChunks);
        else if constexpr (LONG || PAIR) return min(kGroupChunks, chunks - first_chunk(unit));
        else return chunks;
    };
    unsigned char* const b_area = smem + (size_t)a.stages * OpA::kBytes;
    auto load_w = [&](OpB& op, int t, int chunk) {
        if constexpr (P == kGradX) op.load(t, (const TB*)a.W, a.n_out, n0, a.n_in, chunk * kChunk, a.n_out);
        else if constexpr (P != kGradW) op.load(t, (const TB*)a.W, a.n_out, chunk * kChunk, a.n_in, n0, a.n_out);
    };
    if (a.resident && units > 0) {   // all warps bring B in, a chunk for each 256 threads
        for (int k = threadIdx.x / kRoleThreads; k < chunks && warp < kIssuer; k += kIssuer * 32 / kRoleThreads) {
            OpB op;
            load_w(op, threadIdx.x % kRoleThreads, k);
            op.template store<P == kGradX>(threadIdx.x % kRoleThreads, b_area + (size_t)k * OpB::kBytes);
        }
        umma::fence_smem_to_async();
    }
    umma::fence_before_sync();
    __syncthreads();
    umma::fence_after_sync();
    const uint32_t tmem = tmem_slot;

    // A as whole boxes, one thread's work; rows behind the last real one come along, and their results go nowhere
    auto fetch_boxes = [&] {
        int stage = 0;
        uint32_t turn = 0;
        bool ok = true;
        for (int unit = 0; ok && unit < units; ++unit)
            for (int chunk = 0; chunk < chunks; ++chunk) {
                if (turn > 0 && !(ok = fast::mbar_wait(&empty[stage], (turn - 1) & 1, abort_flag, a.status))) break;
                fast::mbar_arrive_expect_tx(&full[stage], OpA::kBytes);
                load_box(umma::smem_addr(smem) + stage * OpA::kBytes, &a.map_a, chunk * kChunk, (int)row_of(unit), &full[stage]);
                if (++stage == a.stages) { stage = 0; ++turn; }
            }
        if (!ok)   // a wait ran out: the copies on their way arrive before the block goes
            for (int i = 0; i < a.stages; ++i)
                if (turn > 0 || i < stage) fast::mbar_wait(&full[i], (i < stage ? turn : turn - 1) & 1, &drain_word, a.status);
    };

    if (warp >= kReaders && warp < kIssuer) {
        // ------------------------------------------------ loaders: memory -> terms -> stages
        const int t = threadIdx.x - kReaders * 32;
        float2 col_sum[2] = {both(0.f), both(0.f)};   // kGradW: of this thread's four columns of gz, the same in every chunk
        if (L::kBoxes && a.boxes) {
            if (warp == kReaders && lane == 0) fetch_boxes();
        } else {
        OpA op_a;
        OpB op_b;
        auto with_a = [&](int unit, int chunk, auto&& f) {   // the block of A that a chunk takes
            if constexpr (P == kGradW) f((const TA*)a.x, (int64_t)a.n_in, (chunk_begin + (int64_t)unit * kGroupChunks + chunk) * kChunkRows, m0, a.n_in);
            else if constexpr (P == kGradX) f((const TA*)a.gz, (int64_t)a.ld_gz, row_of(unit), (first_chunk(unit) + chunk) * kChunk, a.ld_gz);
            else f((const TA*)a.x, (int64_t)a.n_in, row_of(unit), (first_chunk(unit) + chunk) * kChunk, a.n_in);
        };
        auto load_a = [&](int unit, int chunk) {
            if constexpr (!L::kAsyncA)
                with_a(unit, chunk, [&](const TA* from, int64_t ld, int64_t row0, int col0, int col_end) { op_a.load(t, from, ld, row0, real, col0, col_end); });
        };
        auto load_b = [&](int unit, int chunk) {
            if constexpr (P == kGradW) op_b.load(t, (const TB*)a.gz, a.ld_gz, (chunk_begin + (int64_t)unit * kGroupChunks + chunk) * kChunkRows, real, n0, a.ld_gz);
            else load_w(op_b, t, first_chunk(unit) + chunk);
        };
        if (units > 0) {
            load_a(0, 0);
            if (!a.resident) load_b(0, 0);
        }
        const int lag = L::kAsyncA ? min(a.stages - 1, 3) : 0;   // chunks of cp.async on their way behind the newest
        int stage = 0, late = 0, unreported = 0;
        uint32_t turn = 0;
        bool ok = true;
        auto report = [&] {   // the oldest stage that has not been handed over
            umma::fence_smem_to_async();
            __syncwarp();
            if (lane == 0) fast::mbar_arrive(&full[late]);
            late = late + 1 == a.stages ? 0 : late + 1;
            --unreported;
        };
        for (int unit = 0; ok && unit < units; ++unit) {
            const int n_chunks = chunks_of(unit);
            for (int chunk = 0; chunk < n_chunks; ++chunk) {
                if (turn > 0 && !(ok = fast::mbar_wait(&empty[stage], (turn - 1) & 1, abort_flag, a.status))) break;
                unsigned char* const to = smem + (size_t)stage * OpA::kBytes;
                if constexpr (L::kAsyncA)
                    with_a(unit, chunk, [&](const TA* from, int64_t ld, int64_t row0, int col0, int col_end) {
                        copy_async<P == kGradW ? kChunkRows : kTileRows, P == kGradW ? kTileRows : kChunk>(t, umma::smem_addr(to), from, ld, row0, real, col0, col_end);
                    });
                else op_a.store(t, to);
                if (!a.resident) {
                    op_b.template store<P == kGradX>(t, b_area + (size_t)stage * OpB::kBytes);
                    if constexpr (P == kGradW) {
                        if (a.want_sums && m0 == 0)
#pragma unroll
                            for (int i = 0; i < OpB::kItems; ++i) op_b.q[i].add_to(col_sum);
                    }
                }
                if constexpr (L::kAsyncA) async_commit();
                if (++unreported > lag) {
                    if constexpr (L::kAsyncA) async_wait(lag);
                    report();
                }
                const bool more = chunk + 1 < n_chunks;
                if (more || unit + 1 < units) {
                    load_a(more ? unit : unit + 1, more ? chunk + 1 : 0);
                    if (!a.resident) load_b(more ? unit : unit + 1, more ? chunk + 1 : 0);
                }
                if (++stage == a.stages) { stage = 0; ++turn; }
            }
        }
        if constexpr (L::kAsyncA) async_wait(0);
        while (ok && unreported > 0) report();
        }
        if constexpr (P == kGradW) {
            if (a.want_sums && m0 == 0) {
                const int across = t % OpB::kAcross, group = t / OpB::kAcross;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    column_sums[group * NT + across * 4 + 2 * j] = col_sum[j].x;
                    column_sums[group * NT + across * 4 + 2 * j + 1] = col_sum[j].y;
                }
                asm volatile("bar.sync 1, %0;" ::"n"(kRoleThreads) : "memory");
                if (t < NT && n0 + t < a.n_out) {
                    float sum = 0.f;
                    for (int r = 0; r < OpB::kRows; ++r) sum += column_sums[r * NT + t];
                    const int range = blockIdx.x / (a.n_tiles * a.m_tiles);
                    if (a.shares) a.shares[(size_t)(range + 1) * ((size_t)a.n_in * a.n_out + a.n_out) - a.n_out + n0 + t] = sum;
                    else if (a.grad_b) ((T*)a.grad_b)[n0 + t] = from_float<T>(sum);
                }
            }
        } else if (P != kSlope && real < a.rows) {
            // zero rows behind the last real one
            const int width = P == kGradX ? a.n_in : a.n_out;
            T* const out = (T*)a.out;
            for (int64_t i = real * width + blockIdx.x * (int64_t)kRoleThreads + t; i < a.rows * width; i += (int64_t)gridDim.x * kRoleThreads)
                out[i] = from_float<T>(0.f);
        }
    } else if (warp == kIssuer) {
        // ------------------------------------------------ tensor cores
        if (lane == 0) {
            const uint32_t a_addr = umma::smem_addr(smem), b_addr = umma::smem_addr(b_area);
            constexpr uint32_t a_step = L::kA_mn ? 2048 : 32, b_step = L::kB_mn ? 2048 : 32;
            constexpr uint32_t one = idesc_bf16(kTileRows, NT, L::kA_mn, L::kB_mn);
            constexpr uint32_t two = idesc_bf16(kTileRows, 2 * NT <= 256 ? 2 * NT : NT, L::kA_mn, L::kB_mn);
            int stage = 0;
            uint32_t turn = 0;
            bool ok = true;
            for (int unit = 0; ok && unit < units; ++unit) {
                const int n_chunks = chunks_of(unit);
                const int set = unit % L::kUnits;
                if (unit >= L::kUnits && !(ok = fast::mbar_wait(&tile_empty[set], (unit / L::kUnits - 1) & 1, abort_flag, a.status))) break;
                const uint32_t d = tmem + (uint32_t)(set * L::kSets * NT);
                for (int chunk = 0; chunk < n_chunks; ++chunk) {
                    if (!(ok = fast::mbar_wait(&full[stage], turn & 1, abort_flag, a.status))) break;
                    umma::fence_after_sync();
                    const uint32_t pa = a_addr + stage * OpA::kBytes, pb = b_addr + (a.resident ? first_chunk(unit) + chunk : stage) * OpB::kBytes;
                    int steps = L::kRows / 16;   // those that hold anything
                    if constexpr (P != kGradW) steps = min(steps, ((P == kGradX ? a.n_out : a.n_in) - (first_chunk(unit) + chunk) * kChunk + 15) / 16);
                    for (int k = 0; k < steps; ++k) {
                        const uint32_t add = chunk > 0 || k > 0;   // (else the accumulators are overwritten)
                        auto da = [&](int term) { return swizzled_desc(pa + term * OpA::kTermBytes + k * a_step, L::kRows * 128, 1024); };
                        auto db = [&](int term) { return swizzled_desc(pb + term * OpB::kTermBytes + k * b_step, L::kRows * 128, 1024); };
                        if constexpr (kTermsA == 3) {
                            mma_bf16(d, da(0), db(0), two, add);         // hi [hi | mid]
                            mma_bf16(d + NT, da(1), db(0), one, 1);
                            mma_bf16(d + NT, da(1), db(1), one, 1);
                            mma_bf16(d + NT, da(0), db(2), one, 1);
                            mma_bf16(d + NT, da(2), db(0), one, 1);
                        } else {
                            mma_bf16(d, da(0), db(0), one, add);
                            if constexpr (kTermsA == 2) mma_bf16(d, da(1), db(0), one, 1);
                            if constexpr (kTermsB == 2) mma_bf16(d, da(0), db(1), one, 1);
                        }
                    }
                    umma::commit(&empty[stage]);
                    if (++stage == a.stages) { stage = 0; ++turn; }
                }
                if (ok) umma::commit(&tile_full[set]);
            }
            // everything issued is over before tensor memory goes back, also after a wait that ran out
            umma::commit(&drain);
            fast::mbar_wait(&drain, 0, &drain_word, a.status);
        }
        __syncwarp();
    } else {
        // ------------------------------------------------ readers: accumulators -> registers -> memory
        const int first = (warp >> 2) * kWarpColumns, quarter = warp & 3;   // 32 rows and kWarpColumns columns
        constexpr int kSums = P == kGradW || LONG ? kWarpColumns / 8 : 1;
        Quads sums[kSums];
#pragma unroll
        for (int i = 0; i < kSums * 4; ++i) sums[i >> 2].p[i >> 1 & 1][i & 1] = both(0.f);
        // What the results meet in memory, residual or grad_y, is fetched before the tile is waited for: kSlots groups of 16 columns
        // (as many as the registers hold), the others as these become free.
        constexpr bool kMeets = P == kForward || P == kSlope;
        constexpr int kGroups = kWarpColumns / 16, kSlots = !kMeets ? 1 : sizeof(T) == 4 ? 2 : kGroups;
        Quad<T> meets[kSlots][2][2];
        const int width = P == kGradX ? a.n_in : a.n_out;
        const int f0 = n0 + first + 4 * (lane & 3);               // first of this lane's four features in the first group
        const T* const meet = (const T*)(P == kForward ? a.residual : a.grad_y);
        for (int unit = 0; unit < units; unit += PAIR ? 2 : 1) {
            const int set = unit % L::kUnits;
            const int64_t row0 = row_of(unit) + quarter * 32 + lane / 4;
            const bool whole = !LONG || (unit + 1) % chains == 0;   // this unit finishes the tile
            auto fetch = [&](int c) {
                if constexpr (kMeets)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        load_quad<VO>(meets[c % kSlots][r >> 1][r & 1], meet + (row0 + 8 * r) * width + f0 + 16 * c,
                                       row0 + 8 * r < real ? width - f0 - 16 * c : 0);
            };
            if (kMeets && meet && whole)
#pragma unroll
                for (int c = 0; c < kSlots; ++c) fetch(c);
            const int phase = unit / L::kUnits & 1;
            if (!fast::mbar_wait(&tile_full[set], phase, abort_flag, a.status)) break;
            if (PAIR && !fast::mbar_wait(&tile_full[set + 1], phase, abort_flag, a.status)) break;
            umma::fence_after_sync();
#pragma unroll
            for (int c = 0; c < kGroups; ++c) {
                const int col = first + 16 * c;                   // of the tile
                const int f = f0 + 16 * c;
                if (P != kGradW && n0 + col >= width) break;
#pragma unroll
                for (int h = 0; h < 2; ++h) {                     // 16 of the warp's 32 lanes of tensor memory
                    const uint32_t taddr = tmem + ((uint32_t)(quarter * 32 + h * 16) << 16) + (uint32_t)(set * L::kSets * NT + col);
                    Quads v;
                    __syncwarp();
                    tmem_ld_quads(taddr, v);
                    if constexpr (L::kSets == 2) {
                        Quads u;
                        tmem_ld_quads(taddr + NT, u);
                        umma::tmem_ld_wait();
                        add_quads(v, u);
                        if constexpr (PAIR)
#pragma unroll
                            for (int k = 2; k < 4; ++k) {
                                tmem_ld_quads(taddr + k * NT, u);
                                umma::tmem_ld_wait();
                                add_quads(v, u);
                            }
                    } else {
                        umma::tmem_ld_wait();
                    }
                    if constexpr (LONG) {
                        add_quads(sums[c * 2 + h], v);
                        if (!whole) continue;
                        v = sums[c * 2 + h];
#pragma unroll
                        for (int i = 0; i < 4; ++i) sums[c * 2 + h].p[i >> 1][i & 1] = both(0.f);
                    }
                    if constexpr (P == kGradW) {
                        add_quads(sums[c * 2 + h], v);
                    } else {
#pragma unroll
                        for (int s = 0; s < 2; ++s) {
                            const int64_t row = row0 + h * 16 + s * 8;
                            float2 (&z)[2] = v.p[s];
                            if constexpr (kMeets) {
                                const float4 b = *reinterpret_cast<const float4*>(bias + col + 4 * (lane & 3));
                                z[0] = __fadd2_rn(z[0], make_float2(b.x, b.y));
                                z[1] = __fadd2_rn(z[1], make_float2(b.z, b.w));
                            }
                            if (row >= real) continue;
                            if constexpr (P == kForward) {
                                activate_as<ACT, T>(z);
                                if (meet) meets[c % kSlots][h][s].add_to(z);
                            }
                            if constexpr (P == kSlope) {
                                float2 g[2] = {both(0.f), both(0.f)};
                                meets[c % kSlots][h][s].add_to(g);
                                times_slope_as<ACT, T>(g, z);
                                store_quad<true>((float*)a.out + row * a.ld_gz + f, g, a.ld_gz - f);   // (whole vectors: ld_gz)
                            } else {
                                store_quad<VO>((T*)a.out + row * width + f, z, width - f);
                            }
                        }
                    }
                }
                if (kMeets && meet && whole && c + kSlots < kGroups) fetch(c + kSlots);
            }
            umma::fence_before_sync();
            __syncwarp();
            if (lane == 0) {
                fast::mbar_arrive(&tile_empty[set]);
                if (PAIR) fast::mbar_arrive(&tile_empty[set + 1]);
            }
        }
        if constexpr (P == kGradW) {
            const int range = blockIdx.x / (a.n_tiles * a.m_tiles);
            float* const share = a.shares + (size_t)range * ((size_t)a.n_in * a.n_out + a.n_out);   // (none: one range, to grad_W itself)
#pragma unroll
            for (int c = 0; c < kGroups; ++c)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        const int row = m0 + quarter * 32 + h * 16 + s * 8 + lane / 4;
                        const int f = f0 + 16 * c;
                        if (row >= a.n_in) continue;
                        if (a.shares) store_quad<false>(share + (size_t)row * a.n_out + f, sums[c * 2 + h].p[s], a.n_out - f);
                        else if (a.grad_W) store_quad<false>((T*)a.grad_W + (size_t)row * a.n_out + f, sums[c * 2 + h].p[s], a.n_out - f);
                    }
        }
    }
    umma::fence_before_sync();
    __syncthreads();
    umma::fence_after_sync();
    if (warp == kIssuer) umma::tmem_dealloc(tmem, L::kColumns);
    if (beside) fast::grid_dependency_wait();
}

}  // namespace layer
}  // namespace e3j
