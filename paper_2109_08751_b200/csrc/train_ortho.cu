// A matrix update orthogonalised by Newton-Schulz products on the tensor cores (sm_100a).
//
// With m the smaller side, X (m x n) = U / (|U| + eps), tall matrices transposed on the way in and
// out.  Each step of the iteration is three products with fp32 accumulators:
//   Gram    A = X X^T            m x m, symmetric
//   Poly    P = b A + c A A + d I   symmetric
//   Apply   X' = (a - d) X + P X
// Only tiles that reach the diagonal or lie above it are computed for A and P; their epilogue
// writes the mirror image too.
//
// Precision.  Operands are fp16 pairs hi + lo with power-of-two scales; 22 bits.  One product a
// step (16-bit matrices): the tensor cores see hi alone, 11 bits, but the term (a - d) X, through
// which the small singular values grow 3.4-fold a step, is formed from hi + lo, and in the first
// step X is U itself (16-bit inputs are exact in hi; 1 / |U| is folded into the epilogues).  With
// rounded X in that term the result of a low-rank gradient is 1-2 % off, with the pair 0.1 %; random
// matrices are 0.12 % off (from 1000 on a side; 64 x 64 0.19 %), where rounding to bf16 is 0.17 %.  Three products (32-bit matrices): hi hi + hi lo + lo hi, and that
// term from an fp32 copy of X, which hi + lo would cut to 22 bits: 1e-6 (low rank
// up to 7e-6 at 64 x 64, where plain 32-bit arithmetic is 1.4e-5 off).  The shift d = -3/4 (b + c) takes
// most of P's diagonal out of its rounding.  With one product it is for the last step alone: in earlier
// ones it would feed the rounding of hi back into small singular values.
//
// Operations are the floor of large matrices: 4096 x 8192 bf16 2.1 ms, 1145 TFLOP/s at the power limit, the tensor
// pipe busy for 74-81 % of the products' time (shared memory bounds it, see the tiles).  Small ones are bound by the launch
// that each product is: 4 x 256 x 256 104 us, 6 us a product, of which 1.3 until the kernel before has ended
// for this one to see, 1.1 until the first tile is in, 0.6-0.9 multiplying, 2.5 writing out.
#include <cuda.h>
#include <math.h>
#include <string.h>

#include <new>
#include <vector>

#include "train_common.cuh"

using namespace spb;

namespace {

enum { kGram = 0, kPoly = 1, kApply = 2, kLast = 3 };

// ---- tile geometry ------------------------------------------------------------------------------
// A pair of CTAs (cta_group::2) makes a tile of 256 x kN: each holds 128 rows of A, half of B and, in
// its tensor memory, 128 rows of the accumulator.  An SM takes in about 64 bytes a clock; alone a CTA
// would need 96 for 128 x 256 (measured: two thirds of the pair's rate).
constexpr int kTileM = 256, kTileK = 64;
constexpr int kABytes = kTileM / 2 * kTileK * 2;
// Of the epilogue: warps, columns a warp has, stages, shared memory.  One product: 16 warps, each takes
// its columns from tensor memory block by block.  Three: 8 warps with their columns' sums in registers.
template <bool kThree>
constexpr int kOutWarps = kThree ? 8 : 16;
template <bool kThree>
constexpr int kThreads = 64 + 32 * kOutWarps<kThree>;  // warp 0 loads, warp 1 multiplies, the others write out
template <bool kThree>
constexpr int kRing = kThree ? 196608 : 163840;        // 4 stages of 48 KiB; 5 of 32 or 6 of 24
template <bool kThree>
constexpr int kSmem = kRing<kThree> + kOutWarps<kThree> * 32 * 32 * 4 + 1024;  // ring, a block for each warp, alignment
// The tensor cores cut each partial sum towards zero: over K = 4096 a relative error of 1e-5, which
// three products of 32-bit matrices would not survive.  They hand over every few blocks of K to a sum
// rounded in registers: every block where the result is then taken from something of its own size (Poly,
// Apply), every second for Gram; random 256 x 4096 2.0e-6 off, with every second throughout 2.9e-6 (plain
// 32-bit arithmetic: 1.9e-6), for which 1024 x 4096 x 2 takes 745 us and not 632.  Results of 16 bits of 16-bit
// matrices do with every eighth (three products of 1024 x 4096 bf16 into 32-bit weights: 4.0e-6 off that way).
constexpr int flush_blocks(int op, bool full) { return !full ? 8 : op == 0 ? 2 : 1; }
constexpr int kNormParts = 512;                         // CTAs a matrix's norm is summed by
constexpr float kScaleX = 4096.0f, kScaleP = 1024.0f;   // X and A, P are held times these
constexpr unsigned long long kWaitNs = 2000000000ull;   // a wait inside the kernel gives up after this

// ---- PTX ----------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t n) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(n) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, 0x989680;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}
__device__ __forceinline__ unsigned long long now_ns() {
    unsigned long long t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    return t;
}
// Bounded: false once the time is up or another role of the CTA gave up.  For one lane.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile uint32_t* gave_up,
                                         unsigned long long limit) {
    if (bar_try(bar, parity)) return true;
    const unsigned long long until = now_ns() + limit;
    while (!bar_try(bar, parity)) {
        if (*gave_up) return false;
        if (now_ns() > until) {
            *gave_up = 1;
            return false;
        }
    }
    return true;
}
// The same for a whole warp: all lanes get one answer.  Each by itself could see the time run out a look before or
// after another, and what follows a wait (elect, tensor memory) takes all lanes of the warp.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile uint32_t* gave_up,
                                          unsigned long long limit) {
    if (__all_sync(kAllLanes, bar_try(bar, parity))) return true;
    const unsigned long long until = now_ns() + limit;
    while (!__all_sync(kAllLanes, bar_try(bar, parity))) {
        if (__any_sync(kAllLanes, *gave_up || now_ns() > until)) {
            *gave_up = 1;
            return false;
        }
    }
    return true;
}
// Arrival at the barrier at the same place in the pair's first CTA.
__device__ __forceinline__ void bar_arrive_first(uint32_t bar) {
    asm volatile(
        "{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %0, 0;\n\t"
        "mbarrier.arrive.release.cluster.shared::cluster.b64 _, [a];\n\t}" ::"r"(bar)
        : "memory");
}
// A copy into this CTA's shared memory that reports to the barrier of the pair's first CTA (the bit
// that tells the two apart cleared in the barrier's address).
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y, int z) {
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes "
        "[%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
        "l"(map), "r"(bar & 0xfeffffffu), "r"(x), "r"(y), "r"(z)
        : "memory");
}
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(p));
    return p != 0;
}
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Shared-memory operand of 128-byte swizzled rows.  K-major: groups of 8 rows `sbo` apart.  MN-major:
// blocks of 64 elements `lbo` apart, groups of 8 k `sbo` apart.
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, uint32_t lbo, uint32_t sbo) {
    return (uint64_t)((addr & 0x3ffff) >> 4) | ((uint64_t)(lbo >> 4) << 16) | ((uint64_t)(sbo >> 4) << 32) |
           (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ void mma_f16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add)
        : "memory");
}
// Arrives at the barrier at this place in both CTAs once the products issued so far are done.
__device__ __forceinline__ void mma_commit(uint32_t bar) {
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
        "h"((uint16_t)3)
        : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_load16(uint32_t addr, float (&v)[16]) {
    uint32_t r[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr)
        : "memory");
#pragma unroll
    for (int i = 0; i < 16; i++) v[i] = __uint_as_float(r[i]);
}

// ---- arguments ----------------------------------------------------------------------------------

// A user's matrix: element (r, c) of matrix b at p[b * stride + r * ld + c], seen transposed where
// the plan works on the transpose.
struct Mat {
    void* p;
    int64_t ld, stride;
    int type;
    bool wide;  // every row starts on a multiple of 16 bytes
};

struct ProductArgs {
    int M, N, K;            // of the product
    int flush;              // three products: blocks of K that an accumulator takes
    int n_tiles;            // tiles of one matrix, listed in `tiles` as (row tile << 16 | column tile)
    int total;              // tiles of all matrices
    const uint32_t* tiles;
    const float* q;         // per matrix: true X per stored X of the first step
    int first;              // first step: X is the scaled update
    float a, b, c, d;       // coefficients of the step, d already taken off a
    // hi and lo of: the epilogue's addend (Poly: A; Apply: X) and of the result; pitch in elements
    const __half *in_hi, *in_lo;
    __half *out_hi, *out_lo;
    const float* in_full;   // three products: X in fp32, in and out
    float* out_full;
    int64_t ld_in, ld_out, z_in, z_out;  // z: elements between matrices
    // last step: the result, or the weights it updates
    Mat out, weight;
    int transposed, muon;
    float keep, rate;       // W' = keep W - rate X
    uint32_t* status;
    unsigned long long limit;  // ns that a wait inside the kernel may take
    int withhold;              // test of that: finished accumulators are not announced
};

// Four values of a row, the first n of them inside the matrix; `wide`: every row starts on a multiple
// of 16 bytes and c on a multiple of four elements, so that four values are 8 or 16 aligned bytes.
template <typename T>
__device__ __forceinline__ void read4(const T* p, bool wide, int n, float (&v)[4]) {
    if (wide && n >= 4) {
        const Pack<T, 4> k = *reinterpret_cast<const Pack<T, 4>*>(p);
#pragma unroll
        for (int i = 0; i < 4; i++) v[i] = to_float(k.v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; i++) v[i] = i < n ? to_float(p[i]) : 0.0f;
    }
}
template <typename T>
__device__ __forceinline__ void write4(T* p, bool wide, int n, const float (&v)[4]) {
    if (wide && n >= 4) {
        Pack<T, 4> k;
#pragma unroll
        for (int i = 0; i < 4; i++) k.v[i] = from_float<T>(v[i]);
        *reinterpret_cast<Pack<T, 4>*>(p) = k;
    } else {
#pragma unroll
        for (int i = 0; i < 4; i++)
            if (i < n) p[i] = from_float<T>(v[i]);
    }
}
__device__ __forceinline__ void write_any(const Mat& m, int z, int64_t r, int64_t c, int n, const float (&v)[4]) {
    const int64_t at = z * m.stride + r * m.ld + c;
    if (m.type == SPARBIT_F32) write4((float*)m.p + at, m.wide, n, v);
    else if (m.type == SPARBIT_BF16) write4((__nv_bfloat16*)m.p + at, m.wide, n, v);
    else write4((__half*)m.p + at, m.wide, n, v);
}
__device__ __forceinline__ void read_any(const Mat& m, int z, int64_t r, int64_t c, int n, float (&v)[4]) {
    const int64_t at = z * m.stride + r * m.ld + c;
    if (m.type == SPARBIT_F32) read4((const float*)m.p + at, m.wide, n, v);
    else if (m.type == SPARBIT_BF16) read4((const __nv_bfloat16*)m.p + at, m.wide, n, v);
    else read4((const __half*)m.p + at, m.wide, n, v);
}
// The last step's result for four elements of a row of the user's matrix.
__device__ __forceinline__ void write_result(const ProductArgs& g, int z, int64_t r, int64_t c, int n, float (&v)[4]) {
    if (g.muon) {
        float w[4];
        read_any(g.weight, z, r, c, n, w);
#pragma unroll
        for (int i = 0; i < 4; i++) v[i] = g.keep * w[i] - g.rate * v[i];
    }
    write_any(g.out, z, r, c, n, v);
}

// A warp's block of a product in shared memory: columns turned by the row's number, so that neither rows
// nor columns meet a bank twice.
constexpr int kBlock = 32;
__device__ __forceinline__ int block_at(int r, int c) { return r * kBlock + (c ^ r); }

// What the epilogue adds to a block: the lane's four elements of every fourth row, as stored - fp16 hi
// and lo, or fp32.  Loaded before the products are done where registers allow.
struct Addend {
    uint4 raw[kBlock / 4];
};
template <int kOp, bool kThree>
__device__ __forceinline__ void load_addend(const ProductArgs& g, int z, int row0, int col0, Addend& d) {
    if (kOp == kGram) return;
    const int lane = threadIdx.x & 31, row = row0 + (lane >> 3), col = col0 + (lane & 7) * 4;
    const int64_t at = z * g.z_in + row * g.ld_in + col;
#pragma unroll
    for (int it = 0; it < kBlock / 4; it++) {
        if (row + it * 4 >= g.M || col >= g.N) continue;
        const int64_t i = at + (int64_t)(it * 4) * g.ld_in;
        if (kOp != kPoly && kThree) {
            d.raw[it] = *reinterpret_cast<const uint4*>(g.in_full + i);
        } else {
            const uint2 hi = *reinterpret_cast<const uint2*>(g.in_hi + i);
            uint2 lo = make_uint2(0u, 0u);
            if (kOp != kPoly || kThree) lo = *reinterpret_cast<const uint2*>(g.in_lo + i);
            d.raw[it] = make_uint4(hi.x, hi.y, lo.x, lo.y);
        }
    }
}
__device__ __forceinline__ void unpack_halves(uint32_t a, uint32_t b, float (&v)[4]) {
    const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&a));
    const float2 q = __half22float2(*reinterpret_cast<const __half2*>(&b));
    v[0] = p.x, v[1] = p.y, v[2] = q.x, v[3] = q.y;
}

// A block of 32 x 32 elements of a product, on its way out: eight lanes to a row, so that rows leave in
// 64-byte runs; then, where its mirror image or transpose goes out (too), the same by columns.  The
// pitches of X, A and P are multiples of 64 elements: four elements that start inside a row may be read
// and written whole (the columns past the matrix are outside the tensor maps).
template <int kOp, bool kThree>
__device__ __forceinline__ void write_block(const ProductArgs& g, float* sm, int z, int row0, int col0, float q,
                                            const Addend& d) {
    constexpr bool kSquare = kOp == kGram || kOp == kPoly, kLows = kOp == kApply || (kSquare && kThree);
    const int lane = threadIdx.x & 31, lr = lane >> 3, lc = (lane & 7) * 4;
    const bool turn = kSquare ? col0 > row0 : kOp == kLast && g.transposed;
#pragma unroll
    for (int it = 0; it < kBlock / 4; it++) {
        const int row = row0 + it * 4 + lr, col = col0 + lc;
        if (row >= g.M || col >= g.N) continue;
        float v[4], x[4], y[4];
#pragma unroll
        for (int i = 0; i < 4; i++) v[i] = sm[block_at(it * 4 + lr, lc + i)];
        if (kOp != kGram) {
            if (kOp != kPoly && kThree) {
                x[0] = __uint_as_float(d.raw[it].x), x[1] = __uint_as_float(d.raw[it].y);
                x[2] = __uint_as_float(d.raw[it].z), x[3] = __uint_as_float(d.raw[it].w);
            } else {
                unpack_halves(d.raw[it].x, d.raw[it].y, x);
                if (kOp != kPoly || kThree) {
                    unpack_halves(d.raw[it].z, d.raw[it].w, y);
#pragma unroll
                    for (int i = 0; i < 4; i++) x[i] += y[i];
                }
            }
        }
        if (kSquare) {
            const float scale = kOp == kGram ? q * q * kScaleP : g.c / kScaleP;  // result held times kScaleP
#pragma unroll
            for (int i = 0; i < 4; i++) {
                v[i] *= scale;
                if (kOp == kPoly) v[i] += g.b * x[i] + (col + i == row ? g.d * kScaleP : 0.0f);
            }
        } else {
            // stored X' = (a stored X + (P X) / kScaleP) * (true per stored) * kScaleX
            const float scale = q * (kOp == kLast ? 1.0f : kScaleX);
#pragma unroll
            for (int i = 0; i < 4; i++) v[i] = (g.a * x[i] + v[i] * (1.0f / kScaleP)) * scale;
        }
        if (turn) {
#pragma unroll
            for (int i = 0; i < 4; i++) sm[block_at(it * 4 + lr, lc + i)] = v[i];
        }
        if (kOp == kLast) {
            if (!turn) write_result(g, z, row, col, g.N - col, v);
        } else {
            const int64_t to = z * g.z_out + row * g.ld_out + col;
            write4(g.out_hi + to, true, 4, v);
            if (kOp == kApply && kThree) write4(g.out_full + to, true, 4, v);
            if (kLows) {
#pragma unroll
                for (int i = 0; i < 4; i++) v[i] -= __half2float(__float2half_rn(v[i]));
                write4(g.out_lo + to, true, 4, v);
            }
        }
    }
    if (!turn) return;
    __syncwarp();
#pragma unroll 4
    for (int it = 0; it < kBlock / 4; it++) {
        const int col = col0 + it * 4 + lr, row = row0 + lc;
        if (row >= g.M || col >= g.N) continue;
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; i++) v[i] = sm[block_at(lc + i, it * 4 + lr)];
        if (kOp == kLast) {
            write_result(g, z, col, row, g.M - row, v);
        } else {
            const int64_t to = z * g.z_out + col * g.ld_out + row;
            write4(g.out_hi + to, true, 4, v);
            if (kLows) {
#pragma unroll
                for (int i = 0; i < 4; i++) v[i] -= __half2float(__float2half_rn(v[i]));
                write4(g.out_lo + to, true, 4, v);
            }
        }
    }
}

// ---- the product kernel -------------------------------------------------------------------------
// Persistent, a pair of CTAs per pair of SMs.  Maps: A hi, A lo, B hi, B lo; boxes of 64 columns x 128
// rows (A) and kN / 2 rows (B of Gram and Poly) or of 64 columns x 64 rows (Apply's B, used MN-major).
template <int kOp, int kN, bool kThree>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads<kThree>, 1)
    product_kernel(const __grid_constant__ CUtensorMap a_hi, const __grid_constant__ CUtensorMap a_lo,
                   const __grid_constant__ CUtensorMap b_hi, const __grid_constant__ CUtensorMap b_lo,
                   const __grid_constant__ ProductArgs g) {
    constexpr bool kSquare = kOp == kGram || kOp == kPoly;
    constexpr int kBBytes = kN / 2 * kTileK * 2, kParts = kThree ? 2 : 1;
    constexpr int kStageBytes = kParts * (kABytes + kBBytes), kStages = kRing<kThree> / kStageBytes;
    constexpr int kSlots = 512 / kN;  // accumulators: products run ahead of the warps that write out
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t bars[2 * kStages + 2 * kSlots];
    __shared__ uint32_t tmem_base;
    __shared__ uint32_t gave_up;
    const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
    // full, drained: in the first CTA, for both; empty, done: in each
    const uint32_t full = smem_u32(bars), empty = full + 8 * kStages, done = empty + 8 * kStages, drained = done + 8 * kSlots;
    const int warp = __shfl_sync(kAllLanes, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; i++) bar_init(full + 8 * i, 1), bar_init(empty + 8 * i, 1);
        for (int i = 0; i < kSlots; i++) bar_init(done + 8 * i, 1), bar_init(drained + 8 * i, 2 * kOutWarps<kThree>);
        gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base)),
                     "r"(512)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
    fence_before();
    __syncthreads();
    cluster_sync();
    fence_after();
    const uint32_t tmem = tmem_base;
    const int blocks = (g.K + kTileK - 1) / kTileK, flush = kThree ? g.flush : blocks;
    const int pair = blockIdx.x / 2, pairs = gridDim.x / 2;
    // the list of tiles and the maps are the plan's own and do not change: read ahead of the wait
    const uint32_t first_rc = g.tiles[pair % g.n_tiles];
    if (threadIdx.x == 0) {
        const CUtensorMap* maps[4] = {&a_hi, &b_hi, &a_lo, &b_lo};
#pragma unroll
        for (int i = 0; i < (kThree ? 4 : 2); i++) asm volatile("prefetch.tensormap [%0];" ::"l"(maps[i]) : "memory");
    }
    pdl_wait();
    pdl_trigger();

    if (warp == 0) {
        if (lane == 0) {
            uint32_t n = 0;  // stages filled so far
            bool ok = true;
            for (int t = pair; t < g.total && ok; t += pairs) {
                const int z = t / g.n_tiles;
                const uint32_t rc = t == pair ? first_rc : g.tiles[t - z * g.n_tiles];
                const int row = (int)(rc >> 16) * kTileM + rank * (kTileM / 2), col = (int)(rc & 0xffff) * kN + rank * (kN / 2);
                for (int s = 0; s < blocks; s++, n++) {
                    const uint32_t st = n % kStages;
                    if (n >= kStages && !bar_wait(empty + 8 * st, (n / kStages - 1) & 1, &gave_up, g.limit)) {
                        ok = false;
                        break;
                    }
                    const int k = s * kTileK;
                    const uint32_t bar = full + 8 * st;
                    uint32_t dst = ring + st * kStageBytes;
                    if (rank == 0) bar_expect(bar, 2 * kStageBytes);
#pragma unroll
                    for (int part = 0; part < kParts; part++) {
                        tma_load(dst, part ? &a_lo : &a_hi, bar, k, row, z);
                        dst += kABytes;
                        if (kSquare) {
                            tma_load(dst, part ? &b_lo : &b_hi, bar, k, col, z);
                        } else {
#pragma unroll
                            for (int i = 0; i < kN / 128; i++)
                                tma_load(dst + i * kTileK * 128, part ? &b_lo : &b_hi, bar, col + i * 64, k, z);
                        }
                        dst += kBBytes;
                    }
                }
            }
            // the products have read every stage, and said so to both CTAs, before either may end
            for (uint32_t i = n > kStages ? n - kStages : 0; i < n && ok; i++)
                ok = bar_wait(empty + 8 * (i % kStages), (i / kStages) & 1, &gave_up, g.limit);
            if (!ok) {  // let the copies under way land before the CTA ends
                const unsigned long long until = now_ns() + 1000000ull;
                while (now_ns() < until) {
                }
            }
        }
    } else if (warp == 1) {
        // The whole warp walks the loop and one lane issues: what is the same for all lanes stays in uniform
        // registers, and a product's issue fits the 64 clocks that one of 256 x 128 x 16 takes.
        if (rank == 0) {
            // fp16 operands, fp32 accumulator, 256 x kN; B MN-major for Apply
            constexpr uint32_t idesc = (1u << 4) | (kSquare ? 0u : 1u << 16) | ((uint32_t)(kN >> 3) << 17) |
                                       ((uint32_t)(kTileM >> 4) << 24);
            constexpr uint32_t kPart = (kABytes + kBBytes) >> 4;  // from hi to lo, in descriptor units
            const uint64_t a0 = smem_desc(ring, 16, 1024);
            const uint64_t b0 = smem_desc(ring + kABytes, kSquare ? 16 : kTileK * 128, 1024);
            uint32_t n = 0, group = 0;
            bool ok = true;
            for (int t = pair; t < g.total && ok; t += pairs) {
                for (int s0 = 0; s0 < blocks && ok; s0 += flush, group++) {
                    const uint32_t slot = group % kSlots;
                    if (group >= kSlots && !warp_wait(drained + 8 * slot, (group / kSlots - 1) & 1, &gave_up, g.limit)) {
                        ok = false;
                        break;
                    }
                    fence_after();
                    const int end = s0 + flush < blocks ? s0 + flush : blocks;
                    for (int s = s0; s < end; s++, n++) {
                        const uint32_t st = n % kStages;
                        if (!warp_wait(full + 8 * st, (n / kStages) & 1, &gave_up, g.limit)) {
                            ok = false;
                            break;
                        }
                        fence_after();
                        const uint64_t at = a0 + st * (kStageBytes >> 4), bt = b0 + st * (kStageBytes >> 4);
                        if (elect_one()) {
                            // lo hi and hi lo before hi hi: the sum is small while they come in, and less is cut off
#pragma unroll
                            for (int seg = kThree ? 2 : 0; seg >= 0; seg--) {
#pragma unroll
                                for (int k = 0; k < kTileK / 16; k++)
                                    mma_f16(tmem + slot * kN, at + (seg == 2 ? kPart : 0) + k * (32 >> 4),
                                            bt + (seg == 1 ? kPart : 0) + k * ((kSquare ? 32 : 2048) >> 4), idesc,
                                            s > s0 || seg < (kThree ? 2 : 0) || k > 0);
                            }
                            mma_commit(empty + 8 * st);
                        }
                        __syncwarp();
                    }
                    if (ok && !g.withhold && elect_one()) mma_commit(done + 8 * slot);
                    __syncwarp();
                }
            }
            // The other CTA's warps arrive at `drained` in this one's shared memory: the last arrivals, which no later
            // product waits for, must have landed before this CTA may end.
            for (uint32_t i = group > kSlots ? group - kSlots : 0; i < group && ok; i++)
                ok = warp_wait(drained + 8 * (i % kSlots), (i / kSlots) & 1, &gave_up, g.limit);
        }
    } else {
        // TMEM lanes go by the warp's number mod 4; the warps of a quarter share the columns
        constexpr int kCols = kN / (kOutWarps<kThree> / 4), kBlocks = kCols / kBlock;
        const int quad = warp & 3, part = (warp - 2) >> 2;
        const uint32_t lanes = (uint32_t)(quad * 32) << 16;
        float* const sm = reinterpret_cast<float*>(smem_raw + (ring - smem_u32(smem_raw)) + kRing<kThree>) +
                          (warp - 2) * (kBlock * kBlock);
        uint32_t group = 0;
        for (int t = pair; t < g.total; t += pairs) {
            const int z = t / g.n_tiles;
            const uint32_t rc = t == pair ? first_rc : g.tiles[t - z * g.n_tiles];
            const int row0 = (int)(rc >> 16) * kTileM + rank * (kTileM / 2) + quad * 32;
            const int col0 = (int)(rc & 0xffff) * kN + part * kCols;
            const float q = g.first ? g.q[z] : 1.0f / kScaleX;
            // blocks below the diagonal are the mirror images of others
            auto wanted = [&](int j) {
                const int col = col0 + j * kBlock;
                return row0 < g.M && col < g.N && !(kSquare && col < row0);
            };
            Addend d[2];
            bool ok = true;
            if constexpr (!kThree) {
                // the addend of the first block travels while the products run, each other's while its
                // predecessor goes out
                if (wanted(0)) load_addend<kOp, kThree>(g, z, row0, col0, d[0]);
                const uint32_t slot = group % kSlots;
                ok = warp_wait(done + 8 * slot, (group / kSlots) & 1, &gave_up, g.limit);
                if (!ok) break;
                fence_after();
#pragma unroll
                for (int j = 0; j < kBlocks; j++) {
                    const int col = col0 + j * kBlock;
                    float v[16];
                    __syncwarp();
#pragma unroll
                    for (int h = 0; h < 2; h++) {
                        tmem_load16(tmem + slot * kN + part * kCols + j * kBlock + h * 16 + lanes, v);
#pragma unroll
                        for (int i = 0; i < 16; i++) sm[block_at(lane, h * 16 + i)] = v[i];
                    }
                    if (j + 1 == kBlocks) fence_before();
                    __syncwarp();
                    if (j + 1 == kBlocks && lane == 0) bar_arrive_first(drained + 8 * slot);
                    if (j + 1 < kBlocks && wanted(j + 1)) load_addend<kOp, kThree>(g, z, row0, col + kBlock, d[(j + 1) & 1]);
                    if (wanted(j)) write_block<kOp, kThree>(g, sm, z, row0, col, q, d[j & 1]);
                }
                group++;
            } else {
                static_assert(kBlocks == 2, "registers for all addends beside the sums");
#pragma unroll
                for (int j = 0; j < kBlocks; j++)
                    if (wanted(j)) load_addend<kOp, kThree>(g, z, row0, col0 + j * kBlock, d[j]);
                float acc[kCols];
#pragma unroll
                for (int i = 0; i < kCols; i++) acc[i] = 0.0f;
                for (int s = 0; s < blocks; s += flush, group++) {
                    const uint32_t slot = group % kSlots;
                    ok = warp_wait(done + 8 * slot, (group / kSlots) & 1, &gave_up, g.limit);
                    if (!ok) break;
                    fence_after();
#pragma unroll
                    for (int j = 0; j < kCols / 16; j++) {
                        float v[16];
                        __syncwarp();
                        tmem_load16(tmem + slot * kN + part * kCols + j * 16 + lanes, v);
#pragma unroll
                        for (int i = 0; i < 16; i++) acc[j * 16 + i] += v[i];
                    }
                    fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive_first(drained + 8 * slot);
                }
                if (!ok) break;
#pragma unroll
                for (int j = 0; j < kBlocks; j++) {
                    if (wanted(j)) {
                        const int col = col0 + j * kBlock;
                        __syncwarp();
#pragma unroll
                        for (int i = 0; i < kBlock; i++) sm[block_at(lane, i)] = acc[j * kBlock + i];
                        __syncwarp();
                        write_block<kOp, kThree>(g, sm, z, row0, col, q, d[j]);
                    }
                }
            }
        }
    }
    __syncthreads();
    if (threadIdx.x == 0 && gave_up) *g.status = 2;
    // Nobody's barriers or tensor memory are needed any more: every remote arrival has been waited for (empty by the
    // loading warps, done by those that write out, drained by the multiplying warp), so that no order is asked of
    // this barrier.  The stores to global memory are left to the kernel's end (4 x 256 x 256 bf16 104 us, waiting for
    // them here 110).
    asm volatile("barrier.cluster.arrive.relaxed.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
    if (warp == 1) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
}

// ---- before the products ------------------------------------------------------------------------

struct PrepareArgs {
    Mat update;                  // U, or the gradient
    const float* mom_in;         // Muon: momentum, null otherwise
    float* mom_out;
    int64_t mom_ld, mom_stride;
    bool mom_wide;
    float mu;
    int nesterov;
    int rows, cols;              // of the user's matrix
    int transposed;
    float eps;
    double* parts;               // [count][kNormParts]
    float* q;                    // [count]
    __half *hi, *lo;
    float* full;                 // three products
    int64_t ld, z;
};

// Four elements of U; and the new momentum where `write`.
__device__ __forceinline__ void update4(const PrepareArgs& g, int z, int64_t r, int c, bool write, float (&u)[4]) {
    const int n = g.cols - c;
    read_any(g.update, z, r, c, n, u);
    if (!g.mom_in) return;
    float m[4];
    const Mat out{g.mom_out, g.mom_ld, g.mom_stride, SPARBIT_F32, g.mom_wide};
    if (write) {
        const Mat in{(void*)g.mom_in, g.mom_ld, g.mom_stride, SPARBIT_F32, g.mom_wide};
        read_any(in, z, r, c, n, m);
#pragma unroll
        for (int i = 0; i < 4; i++) m[i] = g.mu * m[i] + u[i];
        write_any(out, z, r, c, n, m);
    } else {
        read_any(out, z, r, c, n, m);
    }
#pragma unroll
    for (int i = 0; i < 4; i++) u[i] = g.nesterov ? u[i] + g.mu * m[i] : m[i];
}

// Sum of squares of every matrix, in parts; and the new momentum.
__global__ void __launch_bounds__(256) norm_kernel(const __grid_constant__ PrepareArgs g) {
    __shared__ double s[8];
    pdl_wait();
    pdl_trigger();
    const int z = blockIdx.y, across = (g.cols + 3) / 4;
    const int64_t all = (int64_t)g.rows * across;
    double sum = 0.0;
#pragma unroll 4
    for (int64_t i = blockIdx.x * 256 + threadIdx.x; i < all; i += kNormParts * 256) {
        const int64_t r = all <= 0x7fffffff ? (int)i / across : i / across;
        float u[4];
        update4(g, z, r, (int)(i - r * across) * 4, true, u);
        const float four = u[0] * u[0] + u[1] * u[1] + u[2] * u[2] + u[3] * u[3];
        if (four > 1e-30f && four < 1e30f) {
            sum += (double)four;
        } else {  // squares that 32 bits may not hold
#pragma unroll
            for (int k = 0; k < 4; k++) sum += (double)u[k] * (double)u[k];
        }
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(kAllLanes, sum, o);
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 8; i++) sum += s[i];
        g.parts[(int64_t)z * kNormParts + blockIdx.x] = sum;
    }
}

// X of the first step: U times a power of two (2^120 at most) that brings its norm to 2048 .. 4096, as hi + lo, and
// the factor from that to U / (|U| + eps).  Tiles of 64 x 64, transposed through shared memory.
__global__ void __launch_bounds__(256) convert_kernel(const __grid_constant__ PrepareArgs g) {
    __shared__ double s[8];
    __shared__ float tile[64][65];
    pdl_wait();
    pdl_trigger();
    const int z = blockIdx.z;
    double sum = 0.0;
    for (int i = threadIdx.x; i < kNormParts; i += 256) sum += g.parts[(int64_t)z * kNormParts + i];
    const int tx = (threadIdx.x & 15) * 4, ty = threadIdx.x >> 4;
    const int64_t r0 = (int64_t)blockIdx.y * 64;
    const int c0 = blockIdx.x * 64;
    float u[4][4];
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const int64_t r = r0 + ty + i * 16;
        if (r < g.rows && c0 + tx < g.cols) update4(g, z, r, c0 + tx, false, u[i]);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(kAllLanes, sum, o);
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = sum;
    __syncthreads();
    sum = 0.0;
    for (int i = 0; i < 8; i++) sum += s[i];
    const double norm = sqrt(sum);
    const bool fine = norm > 0.0 && norm < INFINITY;
    int e = 0;
    if (fine) frexp(norm, &e);
    e = min(12 - e, 120);
    const float scale = fine ? ldexpf(1.0f, e) : 1.0f;
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0)
        // zeros stay zeros, whatever eps
        g.q[z] = fine ? (float)(1.0 / (ldexp(norm, e) + ldexp((double)g.eps, e))) : norm == 0.0 ? 0.0f : NAN;
    const int rows = g.transposed ? g.cols : g.rows, cols = g.transposed ? g.rows : g.cols;
    if (g.transposed) {
#pragma unroll
        for (int i = 0; i < 4; i++)
#pragma unroll
            for (int k = 0; k < 4; k++) tile[ty + i * 16][tx + k] = u[i][k];
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const int64_t r = (g.transposed ? c0 : r0) + ty + i * 16;
        const int c = (g.transposed ? (int)r0 : c0) + tx;
        if (r >= rows || c >= cols) continue;
        float v[4];
#pragma unroll
        for (int k = 0; k < 4; k++) v[k] = (g.transposed ? tile[tx + k][ty + i * 16] : u[i][k]) * scale;
        const int64_t to = z * g.z + r * g.ld + c;
        write4(g.hi + to, true, 4, v);
        if (g.full) write4(g.full + to, true, 4, v);
#pragma unroll
        for (int k = 0; k < 4; k++) v[k] -= __half2float(__float2half_rn(v[k]));
        write4(g.lo + to, true, 4, v);
    }
}

typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                             const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                             CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

struct Step {
    float a, b, c;
};

int pick_width(int rows, int cols, int count, bool square, bool three, std::vector<uint32_t>& out);
}  // namespace

struct sparbit_ortho_plan_s {
    int count = 0, dtype = 0, products = SPARBIT_PRODUCTS_AUTO;
    size_t rows = 0, cols = 0;
    int m = 0, n = 0;
    bool transposed = false;
    float eps = 0.0f;
    std::vector<Step> steps;
    std::vector<uint32_t> square, wide;  // tile lists: symmetric results, X
    int square_n = 256, wide_n = 256;    // columns of their tiles
    char* work = nullptr;
    int device = -1, sm_count = 0;
    unsigned long long limit = kWaitNs;
    int withhold = 0;
    // tensor maps: boxes of A operands, of B operands, of MN-major B operands
    CUtensorMap xa[2][2], xb[2][2], xn[2][2], ga[2], gb[2], pa[2];  // [buffer][hi, lo]

    int64_t ldx() const { return (int64_t)round_up(n, 64); }
    int64_t ldg() const { return (int64_t)round_up(m, 64); }
    int64_t zx() const { return ldx() * m; }
    int64_t zg() const { return ldg() * m; }
    // By itself one product for bf16 matrices, unless a side is below 128: error and rounding together are then 1.5 to
    // 1.7 times the rounding to bf16 (64 x 90 2.6e-3, 128 x 128 2.3e-3, 1000 and more 2.0e-3; rounding 1.7e-3), and three
    // products cost a third more (64 x 64 99 us against 73, 128 x 128 121 against 88).
    int parts() const {
        if (products != SPARBIT_PRODUCTS_AUTO) return products;
        return dtype == SPARBIT_BF16 && m >= 128 ? 1 : 3;
    }
    void lay_out() {
        square_n = pick_width(m, m, count, true, parts() == 3, square);
        wide_n = pick_width(m, n, count, false, parts() == 3, wide);
    }
    size_t x_bytes() const { return round_up((size_t)count * zx() * 2, 1024); }
    size_t g_bytes() const { return round_up((size_t)count * zg() * 2, 1024); }
    // layout: status, tiles, parts, q | X hi, lo (two buffers) | A hi, lo | P hi, lo | X fp32 (two buffers)
    size_t off_square() const { return 256; }
    size_t off_wide() const { return off_square() + round_up(square.size() * 4, 256); }
    size_t off_parts() const { return off_wide() + round_up(wide.size() * 4, 256); }
    size_t off_q() const { return off_parts() + (size_t)count * kNormParts * 8; }
    size_t off_x() const { return round_up(off_q() + (size_t)count * 4, 1024); }
    size_t off_g() const { return off_x() + 4 * x_bytes(); }
    size_t off_full() const { return off_g() + 4 * g_bytes(); }
    // 1024: alignment of the base
    size_t work_bytes() const { return off_full() + (parts() == 3 ? 4 * x_bytes() : 0) + 1024; }
    char* base() const { return (char*)round_up((size_t)work, 1024); }
    __half* x(int buffer, int lo) const { return (__half*)(base() + off_x() + (size_t)(2 * buffer + lo) * x_bytes()); }
    float* full(int buffer) const {
        return parts() == 3 ? (float*)(base() + off_full() + (size_t)(2 * buffer) * x_bytes()) : nullptr;
    }
    __half* gram(int lo) const { return (__half*)(base() + off_g() + (size_t)lo * g_bytes()); }
    __half* poly(int lo) const { return (__half*)(base() + off_g() + (size_t)(2 + lo) * g_bytes()); }
};

namespace {

int encode(EncodeFn fn, CUtensorMap* map, void* p, int64_t cols, int64_t rows, int64_t count, int64_t ld, int64_t z,
           int box_rows) {
    const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)count};
    const cuuint64_t strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)z * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1}, one[3] = {1, 1, 1};
    const CUresult r = fn(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, p, dims, strides, box, one,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? SPARBIT_OK : record_cuda_error((int)cudaErrorInvalidValue, "cuTensorMapEncodeTiled");
}

bool wide_rows(const void* q, size_t es, size_t ld, size_t stride) {
    return common_alignment((uintptr_t)q | ld * es | stride * es, 16) == 16;
}

// The largest |value| the iteration can reach over singular values 0 .. 1, and whether X, A and P
// stay within what the scaled fp16 operands hold.
bool bounded(const std::vector<Step>& steps) {
    double s = 1.0;
    for (const Step& k : steps) {
        if (!isfinite(k.a) || !isfinite(k.b) || !isfinite(k.c)) return false;
        double next = 0.0, p = 0.0;
        for (int i = 0; i <= 4096; i++) {
            const double v = s * i / 4096, l = v * v, q = k.b * l + k.c * l * l;
            next = fmax(next, fabs(v * (k.a + q)));
            p = fmax(p, fmax(fabs(q), fabs(q - 0.75 * ((double)k.b + k.c))));
        }
        if (!(p <= 48.0) || !(s * s <= 48.0)) return false;
        s = next * 1.02 + 1e-3;  // what roundings add, and between the points
        if (!(s <= 64.0)) return false;
    }
    return true;
}

int ready(const sparbit_ortho_plan_s* p) {
    if (!p->work) return SPARBIT_ERR_WORKSPACE;
    int cur = -1;
    CU(cudaGetDevice(&cur));
    return cur == p->device ? SPARBIT_OK : SPARBIT_ERR_ARG;
}

template <int kOp, int kN, bool kThree>
int launch_product(const sparbit_ortho_plan_s* p, const CUtensorMap& ah, const CUtensorMap& al, const CUtensorMap& bh,
                   const CUtensorMap& bl, const ProductArgs& g, cudaStream_t st) {
    const int pairs = p->sm_count / 2;
    CU(launch(product_kernel<kOp, kN, kThree>, dim3(2 * (g.total < pairs ? g.total : pairs)), dim3(kThreads<kThree>),
              kSmem<kThree>, st,
              ah, al, bh, bl, g));
    return SPARBIT_OK;
}
template <int kOp>
int product(const sparbit_ortho_plan_s* p, const CUtensorMap& ah, const CUtensorMap& al, const CUtensorMap& bh,
            const CUtensorMap& bl, ProductArgs g, cudaStream_t st) {
    constexpr bool kSquare = kOp == kGram || kOp == kPoly;
    const std::vector<uint32_t>& list = kSquare ? p->square : p->wide;
    g.tiles = (const uint32_t*)(p->base() + (kSquare ? p->off_square() : p->off_wide()));
    g.n_tiles = (int)list.size();
    g.total = g.n_tiles * p->count;
    g.status = (uint32_t*)p->base();
    g.limit = p->limit;
    g.withhold = p->withhold;
    g.flush = flush_blocks(kOp, p->dtype == SPARBIT_F32 || g.out.type == SPARBIT_F32);
    const int n = kSquare ? p->square_n : p->wide_n;
    if (p->parts() == 3) return launch_product<kOp, 128, true>(p, ah, al, bh, bl, g, st);
    return n == 256 ? launch_product<kOp, 256, false>(p, ah, al, bh, bl, g, st)
                    : launch_product<kOp, 128, false>(p, ah, al, bh, bl, g, st);
}
template <int kOp>
int allow_smem() {
    CU(cudaFuncSetAttribute(product_kernel<kOp, 128, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem<true>));
    CU(cudaFuncSetAttribute(product_kernel<kOp, 256, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem<false>));
    CU(cudaFuncSetAttribute(product_kernel<kOp, 128, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem<false>));
    return SPARBIT_OK;
}

// Tiles of 256 x n that a product needs: all of rows x cols, or those that reach the diagonal.
void list_tiles(int rows, int cols, int n, bool square, std::vector<uint32_t>& out) {
    out.clear();
    const int tm = (rows + kTileM - 1) / kTileM, tn = (cols + n - 1) / n;
    if (square) {
        for (int i = 0; i < tm; i++)
            for (int j = i * kTileM / n; j < tn; j++) out.push_back((uint32_t)(i << 16 | j));
    } else {
        // column tiles in the outer loop: the pairs that run together share columns of X and walk down P
        for (int j = 0; j < tn; j++)
            for (int i = 0; i < tm; i++) out.push_back((uint32_t)(i << 16 | j));
    }
}
// Width of the tiles, and their list.  A product reads 6 KiB of shared memory for 256 x 128 x 16 and 8 for
// twice that, so the wider tile multiplies 1.3 times as fast; the narrower one fills the GPU where there
// are few: the rule compares rounds of 74 pairs (a B200's) times the width.  (bf16, narrow against wide:
// 4096 x 8192 2.62 ms against 1.94; 4 x 256 x 256 101 us against 156.)  Three products always take the
// narrow one: their sums then fit the registers beside the addends, and four accumulators fit tensor
// memory (1024 x 4096 x 2 633 us against 756; 4096 x 4096 3.59 ms against 3.49; both with sums taken over
// from tensor memory every second block).
int pick_width(int rows, int cols, int count, bool square, bool three, std::vector<uint32_t>& out) {
    std::vector<uint32_t> wide;
    list_tiles(rows, cols, 256, square, wide);
    list_tiles(rows, cols, 128, square, out);
    const double rounds = (double)((wide.size() * count + 73) / 74), more = (double)((out.size() * count + 73) / 74);
    if (three || more * 128 * 1.3 < rounds * 256) return 128;
    out.swap(wide);
    return 256;
}

// prepare: update, momentum and scalars filled in; last: out, weight, muon, keep, rate filled in
int iterate(const sparbit_ortho_plan_s* p, PrepareArgs prep, ProductArgs last, cudaStream_t st) {
    prep.rows = (int)p->rows;
    prep.cols = (int)p->cols;
    prep.transposed = p->transposed;
    prep.eps = p->eps;
    prep.parts = (double*)(p->base() + p->off_parts());
    prep.q = (float*)(p->base() + p->off_q());
    prep.hi = p->x(0, 0);
    prep.lo = p->x(0, 1);
    prep.full = p->full(0);
    prep.ld = p->ldx();
    prep.z = p->zx();
    CU(launch(norm_kernel, dim3(kNormParts, p->count), dim3(256), 0, st, prep));
    CU(launch(convert_kernel, dim3((unsigned)((p->cols + 63) / 64), (unsigned)((p->rows + 63) / 64), p->count),
              dim3(256), 0, st, prep));
    int cur = 0;
    for (size_t i = 0; i < p->steps.size(); i++) {
        const bool end = i + 1 == p->steps.size();
        ProductArgs g = last;
        const Step& k = p->steps[i];
        g.first = i == 0;
        g.q = prep.q;
        g.b = k.b;
        g.c = k.c;
        g.d = end ? -0.75f * (k.b + k.c) : 0.0f;
        g.a = k.a - g.d;
        g.M = g.N = p->m;
        g.K = p->n;
        g.out_hi = p->gram(0);
        g.out_lo = p->gram(1);
        g.ld_out = p->ldg();
        g.z_out = p->zg();
        int e = product<kGram>(p, p->xa[cur][0], p->xa[cur][1], p->xb[cur][0], p->xb[cur][1], g, st);
        if (e != SPARBIT_OK) return e;
        g.K = p->m;
        g.in_hi = p->gram(0);
        g.in_lo = p->gram(1);
        g.ld_in = p->ldg();
        g.z_in = p->zg();
        g.out_hi = p->poly(0);
        g.out_lo = p->poly(1);
        e = product<kPoly>(p, p->ga[0], p->ga[1], p->gb[0], p->gb[1], g, st);
        if (e != SPARBIT_OK) return e;
        g.N = p->n;
        g.in_hi = p->x(cur, 0);
        g.in_lo = p->x(cur, 1);
        g.in_full = p->full(cur);
        g.out_full = p->full(cur ^ 1);
        g.ld_in = g.ld_out = p->ldx();
        g.z_in = g.z_out = p->zx();
        g.out_hi = p->x(cur ^ 1, 0);
        g.out_lo = p->x(cur ^ 1, 1);
        e = end ? product<kLast>(p, p->pa[0], p->pa[1], p->xn[cur][0], p->xn[cur][1], g, st)
                : product<kApply>(p, p->pa[0], p->pa[1], p->xn[cur][0], p->xn[cur][1], g, st);
        if (e != SPARBIT_OK) return e;
        cur ^= 1;
    }
    return SPARBIT_OK;
}

// A batch lies one matrix behind another, or side by side in the rows of one buffer (column blocks).
bool side_by_side(const sparbit_ortho_plan_s* p, size_t ld, size_t stride) {
    return p->count > 1 && stride >= p->cols && stride <= ld && (p->count - 1) * stride + p->cols <= ld;
}
bool bad_layout(const sparbit_ortho_plan_s* p, size_t ld, size_t stride) {
    if (bad_pitch(ld, p->cols, p->rows)) return true;
    if (p->count == 1 || side_by_side(p, ld, stride)) return false;
    return stride < (p->rows - 1) * ld + p->cols || stride > kMostElements / p->count;
}
Region region(const sparbit_ortho_plan_s* p, const void* q, size_t es, size_t ld, size_t stride) {
    // one matrix of wide rows; of many rows, where the stride is a multiple of the pitch; the whole range otherwise
    if (p->count == 1) return {q, p->rows, p->cols * es, ld * es};
    if (side_by_side(p, ld, stride)) return {q, p->rows, ((p->count - 1) * stride + p->cols) * es, ld * es};
    if (stride % ld == 0) return {q, (stride / ld) * (p->count - 1) + p->rows, p->cols * es, ld * es};
    return {q, 1, ((p->count - 1) * stride + (p->rows - 1) * ld + p->cols) * es, 0};
}

}  // namespace

extern "C" {

int sparbit_ortho_plan_create(int count, size_t rows, size_t cols, int dtype, int steps, const float* coefficients,
                              float eps, sparbit_ortho_plan_t** out) {
    if (!out) return SPARBIT_ERR_ARG;
    *out = nullptr;
    if (count < 1 || rows < 1 || cols < 1 || !known_dtype(dtype) || steps < 1 || !(eps >= 0.0f) || !isfinite(eps))
        return SPARBIT_ERR_ARG;
    if (rows > 65536 || cols > 65536 || steps > 64 || count > 4096) return SPARBIT_ERR_LIMIT;
    sparbit_ortho_plan_s* p = new (std::nothrow) sparbit_ortho_plan_s();
    if (!p) return SPARBIT_ERR_NOMEM;
    bool ok = true;
    try {
        for (int i = 0; i < steps; i++)
            p->steps.push_back(coefficients ? Step{coefficients[3 * i], coefficients[3 * i + 1], coefficients[3 * i + 2]}
                                            : Step{3.4445f, -4.7750f, 2.0315f});
        ok = bounded(p->steps);
        p->count = count;
        p->dtype = dtype;
        p->rows = rows;
        p->cols = cols;
        p->transposed = rows > cols;
        p->m = (int)(rows < cols ? rows : cols);
        p->n = (int)(rows < cols ? cols : rows);
        p->eps = eps;
        p->lay_out();
    } catch (const std::bad_alloc&) {
        delete p;
        return SPARBIT_ERR_NOMEM;
    }
    const size_t most = 0x7fffffffu / (size_t)count;
    if (!ok || p->wide.size() > most || p->square.size() > most) {
        delete p;
        return ok ? SPARBIT_ERR_LIMIT : SPARBIT_ERR_ARG;
    }
    *out = p;
    return SPARBIT_OK;
}

int sparbit_ortho_plan_destroy(sparbit_ortho_plan_t* p) {
    delete p;
    return SPARBIT_OK;
}

int sparbit_ortho_plan_set_products(sparbit_ortho_plan_t* p, int products) {
    if (!p || (products != SPARBIT_PRODUCTS_AUTO && products != SPARBIT_PRODUCTS_ONE && products != SPARBIT_PRODUCTS_THREE))
        return SPARBIT_ERR_ARG;
    p->products = products;
    p->work = nullptr;  // the tiles and the workspace's layout go by it
    try {
        p->lay_out();
    } catch (const std::bad_alloc&) {
        return SPARBIT_ERR_NOMEM;
    }
    return SPARBIT_OK;
}

size_t sparbit_ortho_plan_workspace_bytes(const sparbit_ortho_plan_t* p) { return p ? p->work_bytes() : 0; }

int sparbit_ortho_plan_set_workspace(sparbit_ortho_plan_t* p, void* dev, size_t bytes) {
    if (!p) return SPARBIT_ERR_ARG;
    if (!dev || bytes < p->work_bytes() || (uintptr_t)dev % 16) return SPARBIT_ERR_WORKSPACE;
    p->work = nullptr;
    CU(cudaGetDevice(&p->device));
    CU(cudaDeviceGetAttribute(&p->sm_count, cudaDevAttrMultiProcessorCount, p->device));
    int e = allow_smem<kGram>();
    if (e == SPARBIT_OK) e = allow_smem<kPoly>();
    if (e == SPARBIT_OK) e = allow_smem<kApply>();
    if (e == SPARBIT_OK) e = allow_smem<kLast>();
    if (e != SPARBIT_OK) return e;
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult found;
    CU(cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found));
    if (!fn || found != cudaDriverEntryPointSuccess)
        return record_cuda_error((int)cudaErrorNotSupported, "cuTensorMapEncodeTiled");
    p->work = (char*)dev;
    const EncodeFn f = (EncodeFn)fn;
    const int half = p->square_n / 2;
    for (int lo = 0; lo < 2 && e == SPARBIT_OK; lo++) {
        for (int b = 0; b < 2 && e == SPARBIT_OK; b++) {
            e = encode(f, &p->xa[b][lo], p->x(b, lo), p->n, p->m, p->count, p->ldx(), p->zx(), kTileM / 2);
            if (e == SPARBIT_OK) e = encode(f, &p->xb[b][lo], p->x(b, lo), p->n, p->m, p->count, p->ldx(), p->zx(), half);
            if (e == SPARBIT_OK) e = encode(f, &p->xn[b][lo], p->x(b, lo), p->n, p->m, p->count, p->ldx(), p->zx(), kTileK);
        }
        if (e == SPARBIT_OK) e = encode(f, &p->ga[lo], p->gram(lo), p->m, p->m, p->count, p->ldg(), p->zg(), kTileM / 2);
        if (e == SPARBIT_OK) e = encode(f, &p->gb[lo], p->gram(lo), p->m, p->m, p->count, p->ldg(), p->zg(), half);
        if (e == SPARBIT_OK) e = encode(f, &p->pa[lo], p->poly(lo), p->m, p->m, p->count, p->ldg(), p->zg(), kTileM / 2);
    }
    char* base = p->base();
    p->work = nullptr;
    if (e != SPARBIT_OK) return e;
    CU(cudaMemset(base, 0, 256));
    CU(cudaMemcpy(base + p->off_square(), p->square.data(), p->square.size() * 4, cudaMemcpyHostToDevice));
    CU(cudaMemcpy(base + p->off_wide(), p->wide.data(), p->wide.size() * 4, cudaMemcpyHostToDevice));
    CU(cudaDeviceSynchronize());
    p->work = (char*)dev;
    return SPARBIT_OK;
}

int sparbit_ortho_plan_status(sparbit_ortho_plan_t* p) {
    if (!p) return SPARBIT_ERR_ARG;
    const int e = ready(p);
    if (e != SPARBIT_OK) return e;
    CU(cudaDeviceSynchronize());
    uint32_t word = 0;
    CU(cudaMemcpy(&word, p->base(), 4, cudaMemcpyDeviceToHost));
    if (word == 0) return SPARBIT_OK;
    CU(cudaMemset(p->base(), 0, 4));
    return SPARBIT_ERR_TIMEOUT;
}

int sparbit_ortho_plan_set_wait_test(sparbit_ortho_plan_t* p, int withhold, uint64_t timeout_ns) {
    if (!p) return SPARBIT_ERR_ARG;
    p->withhold = withhold != 0;
    p->limit = timeout_ns ? timeout_ns : kWaitNs;
    return SPARBIT_OK;
}

int sparbit_orthogonalize(sparbit_ortho_plan_t* p, const void* update, size_t ld, size_t stride, void* out,
                          size_t out_ld, size_t out_stride, void* stream) {
    if (!p || !update || !out) return SPARBIT_ERR_ARG;
    if (bad_layout(p, ld, stride) || bad_layout(p, out_ld, out_stride)) return SPARBIT_ERR_ARG;
    const size_t es = elem_size(p->dtype);
    const Region ro = region(p, out, es, out_ld, out_stride), rw{p->work, 1, p->work_bytes(), 0};
    if (regions_overlap(ro, region(p, update, es, ld, stride)) || regions_overlap(ro, rw)) return SPARBIT_ERR_ALIAS;
    const int e = ready(p);
    if (e != SPARBIT_OK) return e;
    PrepareArgs prep = {};
    prep.update = Mat{(void*)update, (int64_t)ld, (int64_t)stride, p->dtype, wide_rows(update, es, ld, stride)};
    ProductArgs last = {};
    last.out = Mat{out, (int64_t)out_ld, (int64_t)out_stride, p->dtype, wide_rows(out, es, out_ld, out_stride)};
    last.transposed = p->transposed;
    return iterate(p, prep, last, (cudaStream_t)stream);
}

int sparbit_muon_step(sparbit_ortho_plan_t* p, const sparbit_muon* a, void* stream) {
    if (!p || !a || !a->grad || !a->momentum_in || !a->momentum_out || !a->weight_in || !a->weight_out)
        return SPARBIT_ERR_ARG;
    if (!known_dtype(a->weight_dtype)) return SPARBIT_ERR_ARG;
    if (bad_layout(p, a->grad_ld, a->grad_stride) || bad_layout(p, a->momentum_ld, a->momentum_stride) ||
        bad_layout(p, a->weight_ld, a->weight_stride))
        return SPARBIT_ERR_ARG;
    const size_t ws = elem_size(a->weight_dtype);
    const Region rg = region(p, a->grad, elem_size(p->dtype), a->grad_ld, a->grad_stride),
                 mi = region(p, a->momentum_in, 4, a->momentum_ld, a->momentum_stride),
                 mo = region(p, a->momentum_out, 4, a->momentum_ld, a->momentum_stride),
                 wi = region(p, a->weight_in, ws, a->weight_ld, a->weight_stride),
                 wo = region(p, a->weight_out, ws, a->weight_ld, a->weight_stride), rw{p->work, 1, p->work_bytes(), 0};
    if (regions_overlap(mo, rg) || regions_overlap(wo, rg) || regions_overlap(mo, wi) || regions_overlap(wo, mi) ||
        regions_overlap(mo, wo) || regions_overlap(mo, rw) || regions_overlap(wo, rw) ||
        (a->momentum_in != a->momentum_out && regions_overlap(mi, mo)) ||
        (a->weight_in != a->weight_out && regions_overlap(wi, wo)))
        return SPARBIT_ERR_ALIAS;
    const int e = ready(p);
    if (e != SPARBIT_OK) return e;
    PrepareArgs prep = {};
    prep.update = Mat{(void*)a->grad, (int64_t)a->grad_ld, (int64_t)a->grad_stride, p->dtype,
                      wide_rows(a->grad, elem_size(p->dtype), a->grad_ld, a->grad_stride)};
    prep.mom_in = a->momentum_in;
    prep.mom_out = a->momentum_out;
    prep.mom_ld = (int64_t)a->momentum_ld;
    prep.mom_stride = (int64_t)a->momentum_stride;
    prep.mom_wide = wide_rows(a->momentum_in, 4, a->momentum_ld, a->momentum_stride) &&
                    wide_rows(a->momentum_out, 4, a->momentum_ld, a->momentum_stride);
    prep.mu = a->momentum;
    prep.nesterov = a->nesterov;
    ProductArgs last = {};
    last.out = Mat{a->weight_out, (int64_t)a->weight_ld, (int64_t)a->weight_stride, a->weight_dtype,
                   wide_rows(a->weight_out, ws, a->weight_ld, a->weight_stride)};
    last.weight = Mat{(void*)a->weight_in, (int64_t)a->weight_ld, (int64_t)a->weight_stride, a->weight_dtype,
                      wide_rows(a->weight_in, ws, a->weight_ld, a->weight_stride)};
    last.transposed = p->transposed;
    last.muon = 1;
    last.keep = 1.0f - a->lr * a->weight_decay;
    last.rate = a->lr * a->scale;
    return iterate(p, prep, last, (cudaStream_t)stream);
}

}  // extern "C"
