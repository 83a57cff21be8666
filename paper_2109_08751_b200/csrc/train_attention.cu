// Linear attention with a decay for each head: S_t = d S_{t-1} + k_t^T v_t, o_t = scale q_t S_t, a state of
// keys x values in 32 bits for each head of each sequence.
//
// In chunks of kChunk tokens, with i, j the tokens of a chunk and Z the state in front of it, a pass is
//   out_i = inter d^(i + e) a_i Z + intra sum_{j <= i} d^(i - j) (a_i . b_j) c_j
//   Z'    = d^n Z + gain sum_j d^(n - e - j) b_j^T c_j
// and all that the operator does is made of such passes (a, b, c; time; e; inter, intra, gain):
//   o    q, k, v     forward   e = 1   scale, scale, 1       Z = S
//   dq   do, v, k    forward   e = 1   scale, scale, 1       Z = S^T
//   dv   k, q, do    backward  e = 0   1, scale, scale       Z = d times the gradient of S
//   dk   v, do, q    backward  e = 0   1, scale, scale       the same, transposed
// so that the backward pass is one launch of the same kernel over three passes.  It reads nothing that the
// forward pass left: the states are computed again, which costs one of dq's four products.
//
// Sequences that are too few to fill the GPU are cut into segments: one launch leaves what each segment adds to a
// state, a fold along the segments makes of it the state that enters each, and the main launch follows.  The
// same three steps, with an allgather in the middle, are what ranks do that hold slices of a sequence.
//
// A token and head has to move 4 x size elements and takes 4 keys x values operations in the recurrence, in chunks another
// 2 kChunk x (keys + values): 8 x 4096 tokens, 16 heads of 128 / 128 are 83 us of bytes and 41 of products forward, at
// 1669 TFLOP/s.  What the kernel issues is more, the state's product once for each part of c: 72 us with bf16's four, 51
// with fp16's two, so that the tensor cores' work is near the bytes.  It takes 138 us in bf16 (backward 485, of 145 of bytes).
// In place of either the hand-overs between a chunk's steps bound it, see the kernel.  f32 is bound by plain multiply-adds out of shared memory.
#include <cuda.h>
#include <math.h>

#include <algorithm>
#include <new>
#include <vector>

#include "train_tensor.cuh"

using namespace spb;

namespace {

constexpr int kChunk = 128;    // tokens of a chunk: rows of the tensor cores' tiles
constexpr int kMostSize = 128; // of a head's keys and values
constexpr int kPanel = 16384;  // bytes of 128 tokens x 64 elements of 16 bits: rows of 128 swizzled bytes
constexpr int kSms = 148;

// ---- arguments ----------------------------------------------------------------------------------

// A piece of a sequence that one CTA goes through from end to end.
struct alignas(16) Segment {
    int64_t row0, seq_len;
    int32_t len, seq;
    int32_t slot;  // of a sequence that is cut: where its states lie; -1: it is the whole sequence
    int32_t ends;  // 1: it begins its sequence in time, 2: it ends it
};

struct Pass {
    const void *a, *b, *c;
    int64_t a_ld, b_ld, c_ld;
    void* out;  // null: only the state
    int64_t out_ld;
    int kd, vd;                // sizes of a head's a and b, and of its c and out
    int a_wide, b_wide, c_wide, out_wide;  // bytes that all their rows of a head start on a multiple of, up to 16
    int reverse, e;
    float inter, intra, gain;
    // states: element (key, value) of head h of sequence u at [u * unit + h * kd * vd + key * k_step + value * v_step]
    const float* z_in;         // null: zero
    float* z_out;              // null: not wanted
    float* decay_out;          // [u * unit_out + h]: decay over the whole sequence; null: not wanted
    int64_t unit_in, unit_out;
    int k_step, v_step;
    // of segments of sequences that are cut, in the same way by their slots: what enters them (null: zero), what they add
    const float* slots_in;
    float* slots_out;
    int skip_ends;             // what the last segment of a sequence adds is not wanted
    int tiled, out_tiled;      // whole chunks are copied by the maps; whole tiles of out too
};

// Tensors as rows x (heads x size), in boxes of a chunk x 64 elements.
struct alignas(64) Maps {
    CUtensorMap a[3], b[3], c[3];  // of the passes
    CUtensorMap out[3];            // boxes of 32 rows x the values of a warp that writes out
};

struct Args {
    Pass pass[3];
    int n_passes, full;  // full: passes have outputs
    const Segment* list;
    int total;           // segments x heads x passes
    int heads;
    const float* log_decay;
    uint32_t stage_bytes;
    int stages;
    int early;           // all passes lay their tiles out alike: one may be copied over while others are in use
    uint32_t* status;
    unsigned long long limit;
    int withhold;
};

// log2 of the decay; far enough below any exponent of 32 bits for a decay of 0, and finite, so that no token's own
// part (d^0) becomes 0 times infinity.
__device__ __forceinline__ float log2_decay(const float* log_decay, int h) {
    const float l = log_decay[h] * 1.44269504f;
    return l < -1e4f ? -1e4f : l;
}

// ---- tensor memory ------------------------------------------------------------------------------

// Columns (32 bits of 128 lanes each): scores, then in their place the weights that multiply c; out; the state's
// addition; a ring of pieces of c^T, in parts.
constexpr uint32_t kColScore = 0, kColOut = 128, kColAdd = 256, kColC = 384, kRingCols = 128;
constexpr int kMostSlots = 4;

__device__ __forceinline__ void tmem_load32(uint32_t addr, uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, "
        "%24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tmem_store32(uint32_t addr, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, "
        "%25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(addr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
        "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
        "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}
__device__ __forceinline__ void tmem_store16(uint32_t addr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(addr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void tmem_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// The same for 16 lanes, laid out as the matrices of ldmatrix and stmatrix: a lane has two neighbouring columns of 32
// bits (one of them in the store, of two 16-bit numbers) of rows lane / 4 and lane / 4 + 8.
__device__ __forceinline__ void tmem_load_16x32(uint32_t addr, float* z) {
    uint32_t r[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.16x256b.x4.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr)
        : "memory");
#pragma unroll
    for (int i = 0; i < 16; i++) z[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_store_16x8(uint32_t addr, const uint32_t (&r)[4]) {
    asm volatile("tcgen05.st.sync.aligned.16x128b.x2.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]),
                 "r"(r[3])
                 : "memory");
}
// D += A B of one CTA: both operands in shared memory, or A in tensor memory.
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add)
        : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
        "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)add)
        : "memory");
}
// A box of 128 rows x 64 elements into a panel.
__device__ __forceinline__ void copy_box(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(
                     dst),
                 "l"(map), "r"(bar), "r"(x), "r"(y)
                 : "memory");
}
// A tile of out from shared memory, in a group of its own.
__device__ __forceinline__ void store_box(const CUtensorMap* map, uint32_t src, int x, int y) {
    asm volatile(
        "cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];\n\t"
        "cp.async.bulk.commit_group;" ::"l"(map),
        "r"(src), "r"(x), "r"(y)
        : "memory");
}
// Arrives at the barrier once the products issued so far are done.
__device__ __forceinline__ void mma_done(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void proxy_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ---- 16-bit types on the tensor cores -----------------------------------------------------------

template <typename T>
struct Bits;
template <>
struct Bits<__nv_bfloat16> {
    static constexpr bool kScaled = false;  // the exponents of 32 bits: nothing to scale
    static constexpr int kParts = 4;        // parts that hold a number of 32 bits
    static constexpr uint32_t kFormat = (1u << 7) | (1u << 10);
    // c times weights w1 + w2 + w3 (the leading, the next and the last 8 bits of 32-bit ones), two tokens: the product with
    // w1 as the two numbers that hold its 16 bits, that with w2 as its leading and its last bits, to which w3's is added.
    static __device__ __forceinline__ void parts_of(uint32_t c, const uint4& w, uint32_t (&part)[4]) {
        asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(part[0]) : "r"(c), "r"(w.x));
        asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(part[1]) : "r"(c), "r"(w.x), "r"(part[0] ^ 0x80008000u));
        asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(part[2]) : "r"(c), "r"(w.y));
        asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(part[3]) : "r"(c), "r"(w.y), "r"(part[2] ^ 0x80008000u));
        asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(part[3]) : "r"(c), "r"(w.z), "r"(part[3]));
    }
    static __device__ __forceinline__ void put_weight(uint32_t* table, int token, float w) {
#pragma unroll
        for (int i = 0; i < 3; i++) {
            const __nv_bfloat16 v = __float2bfloat16_rn(w);
            reinterpret_cast<__nv_bfloat16*>(table)[(token >> 1) * 8 + i * 2 + (token & 1)] = v;
            w -= __bfloat162float(v);
        }
    }
    // part 1 of an infinity or a NaN is a NaN, and makes `odd` one
    static __device__ __forceinline__ void note_odd(uint32_t& odd, uint32_t part) {
        asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(odd) : "r"(part), "r"(0u));
    }
    static __device__ __forceinline__ bool is_odd(uint32_t v) { return (v & 0x7fff7fffu) != 0; }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
    static __device__ __forceinline__ float low(uint32_t v) { return __uint_as_float(v << 16); }
    static __device__ __forceinline__ float high(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }
};
template <>
struct Bits<__half> {
    static constexpr bool kScaled = true;
    static constexpr int kParts = 2;
    static constexpr uint32_t kFormat = 0;
    // The leading 11 bits, rounded: two of these hold 22 bits and a sign.
    static __device__ __forceinline__ uint32_t take(float2& x) {
        const uint32_t v = pack(x.x, x.y);
        x = fma2(make_float2(low(v), high(v)), make_float2(-1.0f, -1.0f), x);
        return v;
    }
    static __device__ __forceinline__ bool is_odd(uint32_t v) {
        return (v & 0x7fffu) >= 0x7c00u || (v >> 16 & 0x7fffu) >= 0x7c00u;
    }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        const __half2 v = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
    static __device__ __forceinline__ void put_weight(uint32_t* table, int token, float w) { table[token] = __float_as_uint(w); }
    // the larger of the magnitudes, a NaN being larger than everything
    static __device__ __forceinline__ void note_odd(uint32_t& odd, uint32_t v) {
        const __half2 m = __hmax2_nan(*reinterpret_cast<const __half2*>(&odd), __habs2(*reinterpret_cast<const __half2*>(&v)));
        odd = *reinterpret_cast<const uint32_t*>(&m);
    }
    static __device__ __forceinline__ float low(uint32_t v) { return __half2float(__ushort_as_half((unsigned short)v)); }
    static __device__ __forceinline__ float high(uint32_t v) {
        return __half2float(__ushort_as_half((unsigned short)(v >> 16)));
    }
};

// The power of two that brings `most` to 2^13 .. 2^14, as an exponent: fp16 has few, so rows of its operands are scaled.
// Up to 2^40: rows whose largest number is smaller than that allows make nothing that fp16 holds.
__device__ __forceinline__ int exponent_for(float most) {
    const int e = (int)(__float_as_uint(most) >> 23 & 0xff);
    if (e == 0 || e == 255) return 0;
    const int by = 13 - (e - 127);
    return by > 40 ? 40 : by < -110 ? -110 : by;
}
// The largest of the four lanes that share a row of ldmatrix' matrices.
__device__ __forceinline__ float max_of_row(float v) {
    v = fmaxf(v, __shfl_xor_sync(kAllLanes, v, 1));
    return fmaxf(v, __shfl_xor_sync(kAllLanes, v, 2));
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Warps of a CTA by what they do, in groups of four for tensor memory (whose lanes go by the warp's number mod 4) and
// for the registers, of which each group gets as many as it needs.
constexpr int kWeightWarps = 4, kOutWarps = 8, kStateWarps = 8, kLoadWarps = 2;
constexpr int kFirstOut = kWeightWarps, kFirstState = kFirstOut + kOutWarps, kFirstLoad = kFirstState + kStateWarps,
              kMultiply = kFirstLoad + kLoadWarps, kMultiplyState = kMultiply + 1;
constexpr int kTensorThreads = 32 * (kFirstLoad + 4);
constexpr int kRegisters = 80, kWeightRegisters = 64, kOutRegisters = 88, kStateRegisters = 96, kOtherRegisters = 48;
static_assert(kWeightRegisters + 2 * kOutRegisters + 2 * kStateRegisters + kOtherRegisters <=
                  kTensorThreads / 128 * kRegisters,
              "more registers than the CTA has would be waited for without end");
template <int kCount>
__device__ __forceinline__ void take_registers() {
    if constexpr (kCount > kRegisters) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kCount));
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kCount));
}

// 128 tokens of one tensor's head into panels of swizzled rows, by one warp; tokens from n on and columns from `width`
// on are zero.
template <int kWide, int kPanels>
__device__ __forceinline__ void load_tile(uint32_t dst, const char* src, int64_t pitch, int width, int n) {
    constexpr int kPieces = kPanels * 8, kRows = 32 / kPieces;  // 16-byte pieces of a row, rows of an instruction
    const int lane = threadIdx.x & 31, row0 = lane / kPieces, piece = lane % kPieces;
    const uint32_t to = dst + (piece >> 3) * kPanel + row0 * 128;
    const char* from = src + row0 * pitch + piece * 16;
    const int left = (width - piece * 8) * 2;  // bytes of this piece that the row has
    for (int m = 0; m < kChunk; m += 8) {
#pragma unroll
        for (int y = 0; y < 8; y += kRows, from += kRows * pitch) {
            const int row = m + row0 + y;
            const uint32_t at = to + (m + y) * 128 + (((piece & 7) ^ (row0 + y)) << 4);
            if constexpr (kWide == 16) {
                const int bytes = row < n && left > 0 ? 16 : 0;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(at), "l"(bytes ? from : src), "r"(bytes)
                             : "memory");
            } else if constexpr (kWide >= 4) {
#pragma unroll
                for (int k = 0; k < 16; k += kWide) {
                    const int bytes = row < n && left > k ? kWide : 0;
                    asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(at + k),
                                 "l"(bytes ? from + k : src), "n"(kWide), "r"(bytes)
                                 : "memory");
                }
            } else {
                uint32_t v[4];
#pragma unroll
                for (int k = 0; k < 4; k++) {
                    const unsigned short* p = reinterpret_cast<const unsigned short*>(from + k * 4);
                    v[k] = row < n && left > k * 4 ? p[0] : 0u;
                    if (row < n && left > k * 4 + 2) v[k] |= (uint32_t)p[1] << 16;
                }
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3])
                             : "memory");
            }
        }
    }
}
template <int kPanels>
__device__ __forceinline__ void load_wide(int wide, uint32_t dst, const char* src, int64_t pitch, int width, int n) {
    if (wide == 16) load_tile<16, kPanels>(dst, src, pitch, width, n);
    else if (wide == 8) load_tile<8, kPanels>(dst, src, pitch, width, n);
    else if (wide == 4) load_tile<4, kPanels>(dst, src, pitch, width, n);
    else load_tile<2, kPanels>(dst, src, pitch, width, n);
}
__device__ __forceinline__ void load_any(int wide, uint32_t dst, const char* src, int64_t pitch, int width, int n) {
    if (width <= 64) load_wide<1>(wide, dst, src, pitch, width, n);
    else load_wide<2>(wide, dst, src, pitch, width, n);
}

// What a CTA is working on.
struct Work {
    const Pass* p;
    Segment s;
    int head, chunks;
    float l2;  // log2 of the decay
};
__device__ __forceinline__ Work work_of(const Args& g, int w) {
    Work k;
    const int pass = w % g.n_passes, rest = w / g.n_passes;
    k.p = &g.pass[pass];
    k.s = g.list[rest / g.heads];
    k.head = rest % g.heads;
    if (k.p->skip_ends && (k.s.ends & (k.p->reverse ? 1 : 2))) k.s.len = 0;
    k.chunks = (k.s.len + kChunk - 1) / kChunk;
    k.l2 = log2_decay(g.log_decay, k.head);
    return k;
}
// A chunk's tokens lie in shared and tensor memory in the order of time; a pass against time goes through the chunks
// from the last to the first, of which the first is the one that may have fewer.
__device__ __forceinline__ int tokens_of(const Work& k, int chunk) {
    const int left = k.s.len - chunk * kChunk;
    return left < kChunk ? left : kChunk;
}
__device__ __forceinline__ int64_t first_row(const Work& k, int chunk) {
    const int at = chunk * kChunk;
    return k.s.row0 + (k.p->reverse ? k.s.len - at - tokens_of(k, chunk) : at);
}
// Where a state goes; null where this segment leaves none.
__device__ __forceinline__ bool leaves_state(const Work& k) { return k.s.ends & (k.p->reverse ? 1 : 2); }
__device__ __forceinline__ float* state_out(const Args& g, const Work& k) {
    const Pass& p = *k.p;
    const int64_t size = (int64_t)p.kd * p.vd;
    if (k.s.slot >= 0 && p.slots_out) return p.slots_out + (k.s.slot * (int64_t)g.heads + k.head) * size;
    return p.z_out && leaves_state(k) ? p.z_out + k.s.seq * p.unit_out + k.head * size : nullptr;
}
__device__ __forceinline__ const float* state_in(const Args& g, const Work& k) {
    const Pass& p = *k.p;
    const int64_t size = (int64_t)p.kd * p.vd;
    if (k.s.slot >= 0) return p.slots_in ? p.slots_in + (k.s.slot * (int64_t)g.heads + k.head) * size : nullptr;
    return p.z_in ? p.z_in + k.s.seq * p.unit_in + k.head * size : nullptr;
}
__device__ __forceinline__ void decay_out(const Work& k, const float* log_decay) {
    const Pass& p = *k.p;
    if (p.decay_out && leaves_state(k) && !(k.s.slot >= 0 && p.slots_out))
        p.decay_out[k.s.seq * p.unit_out + k.head] =
            k.s.seq_len ? (float)exp((double)log_decay[k.head] * (double)k.s.seq_len) : 1.0f;
}

// Shared memory: a ring of chunks and Z, then these.
constexpr int kMostStages = 4;
constexpr uint32_t kRing = 14 * kPanel;
struct Tables {
    // of a stage: a and b are there, c is; everything, b and a are free again
    uint64_t full[kMostStages], full_c[kMostStages], empty[kMostStages], used[kMostStages], entered_a[kMostStages];
    uint64_t scored, scaled, weighted, entered, done, c_ready[kMostSlots], c_free[kMostSlots], added, add_free, z_ready, out_free, met;
    uint32_t tmem, gave_up;
    uint32_t bad[2];  // number of the last (every other) chunk whose c holds an infinity or a NaN
    // what a token's part is worth at the end of the chunk: fp16 as floats, bf16 as three numbers for each pair of tokens
    alignas(16) uint32_t left[2 * kChunk];
    // for each warp d^31 .. d^0 (against time d^0 .. d^31), between numbers that are finite
    alignas(16) float powers[32 * (kWeightWarps + 2)];
    // fp16: powers of two that rows of Z and of the weights are held times
    alignas(4) signed char z_exp[2][kMostSize], w_exp[2][kChunk];
};
constexpr uint32_t kTensorSmem = kRing + sizeof(Tables);
static_assert(kTensorSmem <= 232448, "shared memory of a CTA");

// c holds an infinity or a NaN, which a product would carry to the tokens in front of it (times their weight of zero):
// adds the tokens that count for this lane's row one by one, for 32 columns.
template <typename B>
__device__ __forceinline__ void add_by_hand(uint32_t (&r)[32], uint32_t weights, uint32_t c_tile, int b, int row, bool reverse) {
#pragma unroll 1
    for (int j = reverse ? row & ~31 : 0; j <= (reverse ? kChunk - 1 : row | 31); j += 2) {
        uint32_t pair;
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];\n\ttcgen05.wait::ld.sync.aligned;"
                     : "=r"(pair)
                     : "r"(weights + j / 2)
                     : "memory");
#pragma unroll 1
        for (int i = 0; i < 2; i++) {
            const int token = j + i;
            if (reverse ? token < row : token > row) continue;
            const float weight = i ? B::high(pair) : B::low(pair);
#pragma unroll
            for (int x = 0; x < 32; x += 8) {
                const int col = b * 32 + x;
                uint32_t u[4];
                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                             : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3])
                             : "r"(c_tile + (col >> 6) * kPanel + token * 128 + ((((col >> 3) & 7) ^ (token & 7)) << 4)));
#pragma unroll
                for (int y = 0; y < 8; y++) {
                    const float value = y & 1 ? B::high(u[y / 2]) : B::low(u[y / 2]);
                    r[x + y] = __float_as_uint(fmaf(weight, value, __uint_as_float(r[x + y])));
                }
            }
        }
        __syncwarp();
    }
}

// One CTA per SM, its warps in roles: weights, output, state (and the parts of c for it), loads, products.  A chunk is
//   score = a b^T;  its weights W = intra d^(i - j) score, causal, rounded to 16 bits into tensor memory
//   out = a Z (Z rounded to 16 bits in shared memory), scaled by row in tensor memory, + W c
//   add = (c times gain d^(n - e - j))^T b, the scaled c in 16-bit parts that hold its 32 bits: bf16 four, fp16 two
// with Z in registers (16 values x 128 keys a warp).  W and Z are the only roundings to 16 bits on the way: together they
// leave out about 1.4 times as far off as rounding it to its type does.
//
// What bounds it: a chunk of 128 / 128 takes 7,500 cycles, of which the products alone are 4,100 (their operands come from
// shared memory at 64 bytes a cycle), the copies 3,600; the tensor pipe is busy for half of them, the issue slots for 45 %.
// With only loads and hand-overs left the same pass takes 81 us of 138.  Tensor memory holds one out, one set of scores
// and two pieces of c's parts at that size, so that consecutive chunks overlap by half a chunk only.
//
// fp16 has few exponents: rows of W, c^T and Z are held times powers of two that go by their largest elements.
template <typename T>
__global__ void __launch_bounds__(kTensorThreads, 1) attention_tensor_kernel(const __grid_constant__ Args g,
                                                                            const __grid_constant__ Maps maps) {
    using B = Bits<T>;
    constexpr int kParts = B::kParts;
    // tokens of a piece of c^T (with 16 what a piece costs beside its tokens takes over: 156 us for 138), the ring's slots
    constexpr int kPiece = 32, kPieces = kChunk / kPiece, kSlotCols = kParts * kPiece / 2, kSlots = kRingCols / kSlotCols,
                  kAhead = kSlots / 2;
    static_assert(kAhead <= kSlots && kSlots <= kMostSlots);
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    Tables& tab = *reinterpret_cast<Tables*>(smem_raw + kRing);
    const uint32_t ring = smem_u32(smem_raw), z_base = ring + g.stages * g.stage_bytes;
    volatile uint32_t* const gave_up = &tab.gave_up;
    const uint32_t full = smem_u32(tab.full), empty = smem_u32(tab.empty), used = smem_u32(tab.used),
                   full_c = smem_u32(tab.full_c), entered_a = smem_u32(tab.entered_a), scored = smem_u32(&tab.scored),
                   scaled = smem_u32(&tab.scaled), weighted = smem_u32(&tab.weighted), entered = smem_u32(&tab.entered),
                   done = smem_u32(&tab.done), c_ready = smem_u32(tab.c_ready), c_free = smem_u32(tab.c_free),
                   added = smem_u32(&tab.added), add_free = smem_u32(&tab.add_free), z_ready = smem_u32(&tab.z_ready),
                   out_free = smem_u32(&tab.out_free), met = smem_u32(&tab.met);
    const int warp = __shfl_sync(kAllLanes, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < g.stages; i++)
            bar_init(full + 8 * i, 1), bar_init(empty + 8 * i, g.full ? kOutWarps : 1), bar_init(used + 8 * i, 1),
                bar_init(full_c + 8 * i, 1), bar_init(entered_a + 8 * i, 1);
        bar_init(scored, 1), bar_init(scaled, kWeightWarps), bar_init(weighted, kWeightWarps + kOutWarps + kStateWarps);
        bar_init(entered, 1), bar_init(done, 1);
        for (int i = 0; i < kSlots; i++) bar_init(c_ready + 8 * i, kStateWarps), bar_init(c_free + 8 * i, 1);
        bar_init(added, 1), bar_init(add_free, kStateWarps), bar_init(z_ready, kStateWarps), bar_init(out_free, kOutWarps);
        bar_init(met, kStateWarps);
        tab.bad[0] = tab.bad[1] = 0;
        // rows of 128 swizzled bytes go by absolute addresses
        tab.gave_up = ring % 1024 != 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kMultiply) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tab.tmem)), "r"(512)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = tab.tmem;
    pdl_wait();
    pdl_trigger();
    bool ok = *gave_up == 0;
    uint32_t c = 0;  // chunks so far, of all that this CTA works on

    if (warp < kFirstOut) {
        // ---- weights: a token a lane
        take_registers<kWeightRegisters>();
        const int row = warp * 32 + lane;
        const uint32_t lanes = (uint32_t)(warp * 32) << 16;
        float* const powers = tab.powers + 32 + 32 * warp;
        if (warp == 0) tab.powers[lane] = tab.powers[32 * (kWeightWarps + 1) + lane] = 0.0f;
        for (int w = blockIdx.x; w < g.total && g.full && ok; w += gridDim.x) {
            const Work k = work_of(g, w);
            const Pass& p = *k.p;
            __syncwarp();
            powers[lane] = exp2f(k.l2 * (p.reverse ? lane : 31 - lane));
            __syncwarp();
            // blocks of 32 tokens of c whose weights are all wanted: [begin, end); of the warp's own block some are
            const int begin = p.reverse ? warp + 1 : 0, end = p.reverse ? 4 : warp;
            const uint32_t causal = p.reverse ? ~0u << lane : 2u << lane, wanted = p.reverse ? causal : causal - 1;
            for (int chunk = 0; chunk < k.chunks; chunk++, c++) {
                if (!warp_wait(scored, c & 1, gave_up, g.limit)) { ok = false; break; }
                fence_after();
                float up = 1.0f;
                if constexpr (B::kScaled) {
                    float most = 0.0f;
#pragma unroll 1
                    for (int b = min(begin, warp); b < max(end, warp + 1); b++) {
                        uint32_t r[32];
                        tmem_load32(tmem + kColScore + lanes + b * 32, r);
                        const uint32_t look = b == warp ? wanted : ~0u;
#pragma unroll
                        for (int j = 0; j < 32; j++)
                            if (look & (1u << j)) most = fmaxf(most, fabsf(__uint_as_float(r[j])));
                    }
                    const int e = exponent_for(most * fabsf(p.intra));
                    up = power_of_two(e);
                    tab.w_exp[c & 1][row] = (signed char)e;
                    __syncwarp();
                    if (lane == 0) bar_arrive(scaled);
                }
// loops of few instructions: what the kinds of warps execute at a time has to fit the instruction caches.  In this order
// the weights of a block lie over scores that have been read.
#pragma unroll 1
                for (int b = 0; b < 4; b++) {
                    uint32_t out[16];
                    if (b == warp) {
                        uint32_t r[32];
                        tmem_load32(tmem + kColScore + lanes + b * 32, r);
                        const float f = p.intra * up;
                        const float* const own = powers + (p.reverse ? -lane : 31 - lane);
#pragma unroll
                        for (int j = 0; j < 32; j += 2) {
                            // what the score of a token that does not count holds is not looked at
                            const float x = wanted & (1u << j) ? __uint_as_float(r[j]) * (own[j] * f) : 0.0f;
                            const float y = wanted & (2u << j) ? __uint_as_float(r[j + 1]) * (own[j + 1] * f) : 0.0f;
                            out[j / 2] = B::pack(x, y);
                        }
                    } else if (b >= begin && b < end) {
                        uint32_t r[32];
                        tmem_load32(tmem + kColScore + lanes + b * 32, r);
                        // to the block's nearest token
                        const float f = exp2f(k.l2 * (p.reverse ? b * 32 - row : row - b * 32 - 31)) * p.intra * up;
#pragma unroll
                        for (int j = 0; j < 32; j += 4) {
                            const float4 d = *reinterpret_cast<const float4*>(powers + j);  // and from there on
                            const float2 x = mul2(mul2(make_float2(d.x, d.y), make_float2(f, f)),
                                                  make_float2(__uint_as_float(r[j]), __uint_as_float(r[j + 1])));
                            const float2 y = mul2(mul2(make_float2(d.z, d.w), make_float2(f, f)),
                                                  make_float2(__uint_as_float(r[j + 2]), __uint_as_float(r[j + 3])));
                            out[j / 2] = B::pack(x.x, x.y), out[j / 2 + 1] = B::pack(y.x, y.y);
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < 16; j++) out[j] = 0u;
                    }
                    tmem_store16(tmem + kColScore + lanes + b * 16, out);
                }
                tmem_store_wait();
                fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(weighted);
            }
        }
    } else if (warp < kFirstState) {
        // ---- output: a token a lane, half of the values a warp
        take_registers<kOutRegisters>();
        const int quad = warp & 3, half = (warp - kFirstOut) >> 2, row = quad * 32 + lane;
        const uint32_t lanes = (uint32_t)(quad * 32) << 16;
        for (int w = blockIdx.x; w < g.total && g.full && ok; w += gridDim.x) {
            const Work k = work_of(g, w);
            const Pass& p = *k.p;
            const int panels_k = (p.kd + 63) / 64;
            const int all = (p.vd + 31) / 32, share = (all + 1) / 2, b0 = half * share, b1 = min(all, b0 + share);
            const uint32_t pitch = share * 64;  // bytes of a row of the warp's values
            const int turn = share == 2 ? lane & 7 : (lane >> 1) & 3;  // of the 16-byte pieces of this lane's row
            const int pass = (int)(k.p - g.pass);
            for (int chunk = 0; chunk < k.chunks; chunk++, c++) {
                const uint32_t st = c % g.stages, stage = ring + st * g.stage_bytes;
                const int n = tokens_of(k, chunk);
                // of rows behind the last token whatever comes
                const float enter = p.inter * exp2f(k.l2 * (p.e + (p.reverse ? n - 1 - row : row)));
                if (!warp_wait(entered, c & 1, gave_up, g.limit)) { ok = false; break; }
                float rise = enter, down = 1.0f;
                if constexpr (B::kScaled) {
                    if (!warp_wait(scaled, c & 1, gave_up, g.limit)) { ok = false; break; }
                    const int e = tab.w_exp[c & 1][row];
                    rise *= power_of_two(e), down = power_of_two(-e);
                }
                fence_after();
#pragma unroll 1
                for (int b = b0; b < b1; b++) {
                    uint32_t r[32];
                    tmem_load32(tmem + kColOut + lanes + b * 32, r);
#pragma unroll
                    for (int j = 0; j < 32; j += 2) {
                        float2 v = mul2(make_float2(__uint_as_float(r[j]), __uint_as_float(r[j + 1])), make_float2(rise, rise));
                        if constexpr (B::kScaled) {
                            const char2 e = *reinterpret_cast<const char2*>(&tab.z_exp[c & 1][b * 32 + j]);
                            v = mul2(v, make_float2(power_of_two(-e.x), power_of_two(-e.y)));
                        }
                        r[j] = __float_as_uint(v.x), r[j + 1] = __float_as_uint(v.y);
                    }
                    tmem_store32(tmem + kColOut + lanes + b * 32, r);
                }
                tmem_store_wait();
                fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(weighted);
                if (!warp_wait(done, c & 1, gave_up, g.limit)) { ok = false; break; }
                fence_after();
                const bool by_hand = *(volatile uint32_t*)&tab.bad[c & 1] == c + 1;
                // in 16 bits over the tile of c
                const uint32_t own = stage + 2 * panels_k * kPanel + (quad * 2 + half) * 32 * pitch;
                uint32_t v[2][16];
#pragma unroll
                for (int b = 0; b < 2; b++) {
                    if (b0 + b >= b1) break;
                    uint32_t r[32];
                    tmem_load32(tmem + kColOut + lanes + (b0 + b) * 32, r);
                    if (by_hand)
                        add_by_hand<B>(r, tmem + kColScore + lanes, stage + 2 * panels_k * kPanel, b0 + b, row, p.reverse);
#pragma unroll
                    for (int j = 0; j < 16; j++) {
                        float2 x = make_float2(__uint_as_float(r[2 * j]), __uint_as_float(r[2 * j + 1]));
                        if constexpr (B::kScaled) x = mul2(x, make_float2(down, down));
                        v[b][j] = B::pack(x.x, x.y);
                    }
                }
                fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(out_free);
                // once everybody who adds c up has read it
                if (by_hand && !warp_wait(out_free, c & 1, gave_up, g.limit)) { ok = false; break; }
#pragma unroll
                for (int b = 0; b < 2; b++) {
                    if (b0 + b >= b1) break;
#pragma unroll
                    for (int j = 0; j < 4; j++)
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(
                                         own + lane * pitch + (((b * 4 + j) ^ turn) << 4)),
                                     "r"(v[b][4 * j]), "r"(v[b][4 * j + 1]), "r"(v[b][4 * j + 2]), "r"(v[b][4 * j + 3])
                                     : "memory");
                }
                const int rows = min(32, n - quad * 32);
                if (p.out_tiled && rows == 32) {
                    proxy_fence();
                    __syncwarp();
                    if (lane == 0 && b0 < b1) {
                        store_box(&maps.out[pass], own, k.head * p.vd + b0 * 32, (int)first_row(k, chunk) + quad * 32);
                        asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                    }
                    __syncwarp();
                    if (lane == 0) bar_arrive(empty + 8 * st);
                    continue;
                }
                __syncwarp();
                T* const to = (T*)p.out + first_row(k, chunk) * p.out_ld + (int64_t)k.head * p.vd + b0 * 32;
                const int64_t way = p.out_ld;
                const int width = min(p.vd, b1 * 32) - b0 * 32;  // of the warp's values
                if (p.out_wide == 16) {
                    // 4 or 8 lanes to a row
                    const int per_row = share * 4, piece = lane & (per_row - 1), r0 = lane / per_row, step = 32 / per_row;
                    T* q = to + (quad * 32 + r0) * way + piece * 8;
                    if (piece * 8 < width) {
#pragma unroll 4
                        for (int r = r0; r < rows; r += step, q += step * way) {
                            uint32_t u[4];
                            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                                         : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3])
                                         : "r"(own + r * pitch + ((piece ^ (share == 2 ? r & 7 : (r >> 1) & 3)) << 4))
                                         : "memory");
                            *reinterpret_cast<uint4*>(q) = make_uint4(u[0], u[1], u[2], u[3]);
                        }
                    }
                } else {
                    for (int r = 0; r < rows; r++) {
                        T* const q = to + (quad * 32 + r) * way;
                        for (int col = lane; col < width; col += 32) {
                            unsigned short u;
                            asm volatile("ld.shared.u16 %0, [%1];"
                                         : "=h"(u)
                                         : "r"(own + r * pitch + (((col >> 3) ^ (share == 2 ? r & 7 : (r >> 1) & 3)) << 4) + (col & 7) * 2)
                                         : "memory");
                            reinterpret_cast<unsigned short*>(q)[col] = u;
                        }
                    }
                }
                // what was read and written here comes before the next chunk's copies
                proxy_fence();
                __syncwarp();
                if (lane == 0) bar_arrive(empty + 8 * st);
            }
        }
    } else if (warp < kFirstLoad) {
        // ---- the state, and c^T for it: a warp has 16 values.  Of Z a lane has rows lane / 4 and lane / 4 + 8 and every
        // fourth pair of keys - z[4 m ..]: keys 8 m + 2 (lane % 4) and the next of the first row, the same of the second -
        // and of c^T tokens 2 (lane % 4) and the next of every 8, for the same rows
        take_registers<kStateRegisters>();
        const int v0 = (warp & 3) * 32 + ((warp - kFirstState) >> 2) * 16, value = v0 + (lane >> 2);
        const int t = threadIdx.x - 32 * kFirstState;
        const uint32_t lanes = (uint32_t)v0 << 16;
        // where this lane's row of the four 8 x 8 matrices that ldmatrix and stmatrix take lies
        const int matrix = lane >> 3, line = lane & 7;
        const uint32_t z_lane = z_base + (v0 + (matrix & 1) * 8 + line) * 128;
        const uint32_t c_lane = ((matrix >> 1) * 8 + line) * 128 + ((v0 >> 3) + (matrix & 1) >> 3) * kPanel +
                                (((((v0 >> 3) + (matrix & 1)) & 7) ^ line) << 4);
        uint32_t pieces = 0, meetings = 0;
        // a barrier of these warps that gives up like every other wait
        auto meet = [&] {
            __syncwarp();
            if (lane == 0) bar_arrive(met);
            ok = ok && warp_wait(met, meetings++ & 1, gave_up, g.limit);
        };
        for (int w = blockIdx.x; w < g.total && ok; w += gridDim.x) {
            const Work k = work_of(g, w);
            const Pass& p = *k.p;
            const int panels_k = (p.kd + 63) / 64, blocks = (p.kd + 15) / 16 * 2;  // of 8 keys
            const bool there = v0 < p.vd;
            float z[64];
            const float* from = state_in(g, k);
#pragma unroll
            for (int i = 0; i < 64; i++) {
                const int key = (i >> 2) * 8 + (lane & 3) * 2 + (i & 1), v = value + (i & 2) * 4;
                z[i] = from && v < p.vd && key < p.kd ? from[(int64_t)key * p.k_step + (int64_t)v * p.v_step] : 0.0f;
            }
            // rounds Z into shared memory for the products with a
            auto put = [&](uint32_t of) {
                float up[2] = {1.0f, 1.0f};
                if constexpr (B::kScaled) {
                    float most[2] = {0.0f, 0.0f};
#pragma unroll
                    for (int i = 0; i < 64; i++)
                        if ((i >> 2) < blocks)  // what lies behind the last key is nobody's
                            most[(i >> 1) & 1] = fmaxf(most[(i >> 1) & 1], fabsf(z[i]));
#pragma unroll
                    for (int i = 0; i < 2; i++) {
                        const int e = exponent_for(max_of_row(most[i]));
                        if ((lane & 3) == 0) tab.z_exp[of & 1][value + 8 * i] = (signed char)e;
                        up[i] = power_of_two(e);
                    }
                }
                if (there) {
#pragma unroll
                    for (int m = 0; m < 16; m += 2) {
                        if (m >= blocks) break;
                        uint32_t v[4];
#pragma unroll
                        for (int i = 0; i < 4; i++) {
                            float x = z[m * 4 + i * 2], y = z[m * 4 + i * 2 + 1];
                            if constexpr (B::kScaled) x *= up[i & 1], y *= up[i & 1];
                            v[i] = B::pack(x, y);
                        }
                        asm volatile("stmatrix.sync.aligned.m8n8.x4.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(
                                         z_lane + (m >> 3) * kPanel + ((((m & 7) | (matrix >> 1)) ^ line) << 4)),
                                     "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3])
                                     : "memory");
                    }
                }
                proxy_fence();
                __syncwarp();
                if (lane == 0) bar_arrive(z_ready);
            };
            if (g.full && k.chunks) {
                // the chunk before has read its Z
                if (c > 0 && !warp_wait(entered, (c - 1) & 1, gave_up, g.limit)) { ok = false; break; }
                put(c);
            }
            const float* const left = reinterpret_cast<const float*>(tab.left) + (lane & 3) * 2;  // fp16
            const uint4* const pairs = reinterpret_cast<const uint4*>(tab.left) + (lane & 3);     // bf16
            float up[2] = {1.0f, 1.0f};
            uint32_t odd = 0, c_tile = 0;
            // ahead: while a chunk's products are on their way, half of the ring is filled for the next one
            if (k.chunks) c--;
            for (int chunk = k.chunks ? -1 : 0; chunk < k.chunks && ok; chunk++, c++) {
                const float down[2] = {1.0f / up[0], 1.0f / up[1]};
#pragma unroll 1
                for (int i = chunk < 0 ? kPieces - kAhead : 0; i < (chunk + 1 < k.chunks ? kPieces : kPieces - kAhead); i++, pieces++) {
                    const int q = (i + kAhead) % kPieces;
                    // 16 tokens of the warp's values, transposed
                    auto read = [&](int token, uint32_t (&u)[4]) {
                        asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                                     : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3])
                                     : "r"(c_tile + token * 128)
                                     : "memory");
                    };
                    if (i == kPieces - kAhead) {
                        const uint32_t next = c + 1, st = next % g.stages;
                        const int n = tokens_of(k, chunk + 1);
                        if (chunk < 0 || n < kChunk) {  // others are as the one before
                            meet();
                            if (t < kChunk)
                                B::put_weight(tab.left, t, t < n ? p.gain * exp2f(k.l2 * (p.reverse ? t + 1 - p.e : n - p.e - t)) : 0.0f);
                            meet();
                        }
                        if (!ok || !warp_wait(full_c + 8 * st, (next / g.stages) & 1, gave_up, g.limit)) { ok = false; break; }
                        c_tile = ring + st * g.stage_bytes + 2 * panels_k * kPanel + c_lane;
                        odd = 0;
                        if constexpr (B::kScaled) {
                            float m[2] = {0.0f, 0.0f};
                            if (there) {
#pragma unroll 1
                                for (int token = 0; token < kChunk; token += 16) {
                                    uint32_t u[4];
                                    read(token, u);
#pragma unroll
                                    for (int y = 0; y < 4; y++) {
                                        const float2 f = *reinterpret_cast<const float2*>(left + token + (y >> 1) * 8);
                                        m[y & 1] = fmaxf(m[y & 1], fmaxf(fabsf(B::low(u[y]) * f.x), fabsf(B::high(u[y]) * f.y)));
                                    }
                                }
                            }
#pragma unroll
                            for (int y = 0; y < 2; y++) up[y] = power_of_two(exponent_for(max_of_row(m[y])));
                        }
                    }
                    const uint32_t slot = pieces % kSlots;
                    if (pieces >= kSlots && !warp_wait(c_free + 8 * slot, (pieces / kSlots - 1) & 1, gave_up, g.limit)) {
                        ok = false;
                        break;
                    }
                    fence_after();
                    if (there) {
#pragma unroll
                        for (int token = q * kPiece; token < q * kPiece + kPiece; token += 16) {
                            uint32_t part[kParts][4], u[4];
                            read(token, u);
#pragma unroll
                            for (int y = 0; y < 4; y++) {
                                if constexpr (!B::kScaled) {
                                    uint32_t four[4];
                                    B::parts_of(u[y], pairs[token / 2 + (y >> 1) * 4], four);
                                    B::note_odd(odd, four[1]);
#pragma unroll
                                    for (int m = 0; m < kParts; m++) part[m][y] = four[m];
                                } else {
                                    B::note_odd(odd, u[y]);
                                    const float2 f = *reinterpret_cast<const float2*>(left + token + (y >> 1) * 8);
                                    float2 x = mul2(mul2(make_float2(B::low(u[y]), B::high(u[y])), f), make_float2(up[y & 1], up[y & 1]));
#pragma unroll
                                    for (int m = 0; m < kParts; m++) part[m][y] = B::take(x);
                                }
                            }
#pragma unroll
                            for (int y = 0; y < kParts; y++)
                                tmem_store_16x8(tmem + kColC + slot * kSlotCols + y * (kPiece / 2) + token % kPiece / 2 + lanes, part[y]);
                        }
                        tmem_store_wait();
                    }
                    if (q == kPieces - 1 && g.full) {
                        // not more than a chunk ahead of the output, for which the number of a chunk with odd values is left
                        if (c > 0 && !warp_wait(done, (c - 1) & 1, gave_up, g.limit)) { ok = false; break; }
                        if (there && B::is_odd(odd)) *(volatile uint32_t*)&tab.bad[c & 1] = c + 1;
                    }
                    fence_before();
                    __syncwarp();
                    if (lane == 0) {
                        bar_arrive(c_ready + 8 * slot);
                        if (q == kPieces - 1 && g.full) bar_arrive(weighted);
                    }
                }
                if (chunk < 0) continue;
                const int n = tokens_of(k, chunk);
                const float decay = exp2f(k.l2 * n);
                if (!ok || !warp_wait(added, c & 1, gave_up, g.limit)) { ok = false; break; }
                fence_after();
                if (there) {
#pragma unroll
                    for (int b = 0; b < 4; b++) {
                        if (b * 4 >= blocks) break;
                        float v[16];
                        tmem_load_16x32(tmem + kColAdd + lanes + b * 32, v);
#pragma unroll
                        for (int i = 0; i < 16; i += 2) {
                            float2 x = make_float2(v[i], v[i + 1]);
                            if constexpr (B::kScaled) x = mul2(x, make_float2(down[(i >> 1) & 1], down[(i >> 1) & 1]));
                            x = fma2(make_float2(z[b * 16 + i], z[b * 16 + i + 1]), make_float2(decay, decay), x);
                            z[b * 16 + i] = x.x, z[b * 16 + i + 1] = x.y;
                        }
                    }
                }
                fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(add_free);
                if (g.full && chunk + 1 < k.chunks) {
                    if (!warp_wait(entered, c & 1, gave_up, g.limit)) { ok = false; break; }
                    put(c + 1);
                }
            }
            if (!ok) break;
            float* const to = state_out(g, k);
            if (to) {
#pragma unroll
                for (int i = 0; i < 64; i++) {
                    const int key = (i >> 2) * 8 + (lane & 3) * 2 + (i & 1), v = value + (i & 2) * 4;
                    if (v < p.vd && key < p.kd) to[(int64_t)key * p.k_step + (int64_t)v * p.v_step] = z[i];
                }
            }
            if (warp == kFirstState && lane == 0) decay_out(k, g.log_decay);
        }
    } else {
        take_registers<kOtherRegisters>();  // all of the group at one place
        if (warp < kMultiply) {
            // ---- loads: every other chunk each, so that one chunk's copies fly while the other's are waited for
            const uint32_t turn = warp - kFirstLoad;
            for (int w = blockIdx.x; w < g.total && ok; w += gridDim.x) {
                const Work k = work_of(g, w);
                const Pass& p = *k.p;
                const int panels_k = (p.kd + 63) / 64, panels_v = (p.vd + 63) / 64, pass = (int)(k.p - g.pass);
                for (int chunk = 0; chunk < k.chunks; chunk++, c++) {
                    if (c % kLoadWarps != turn) continue;
                    const uint32_t st = c % g.stages, stage = ring + st * g.stage_bytes, bar = full + 8 * st;
                    const uint32_t before = (c / g.stages - 1) & 1;  // parity of this stage's last use
                    const int n = tokens_of(k, chunk);
                    // the chunk that was here before laid its tiles out alike
                    const bool alike = g.full && (g.early ? c >= (uint32_t)g.stages : chunk >= g.stages);
                    const bool tiled = p.tiled && n == kChunk, early = tiled && alike;
                    if (c >= (uint32_t)g.stages && !warp_wait((early ? entered_a : empty) + 8 * st, before, gave_up, g.limit)) {
                        ok = false;
                        break;
                    }
                    // out leaves a stage without waiting for the state's products
                    if (c >= (uint32_t)g.stages && g.full && !early && !warp_wait(used + 8 * st, before, gave_up, g.limit)) {
                        ok = false;
                        break;
                    }
                    const int64_t row = first_row(k, chunk);
                    if (tiled) {
                        // in the order in which the tiles become free: a when its products are done (then b's with it are,
                        // too), b with the state's products, c when out, which goes through its place, has left
                        if (lane == 0) {
                            bar_expect(bar, (g.full ? 2 : 1) * panels_k * kPanel);
                            for (int i = 0; i < panels_k && g.full; i++)
                                copy_box(stage + i * kPanel, &maps.a[pass], bar, k.head * p.kd + i * 64, (int)row);
                        }
                        __syncwarp();
                        if (early && !warp_wait(used + 8 * st, before, gave_up, g.limit)) { ok = false; break; }
                        if (lane == 0)
                            for (int i = 0; i < panels_k; i++)
                                copy_box(stage + (panels_k + i) * kPanel, &maps.b[pass], bar, k.head * p.kd + i * 64, (int)row);
                        __syncwarp();
                        if (early && !warp_wait(empty + 8 * st, before, gave_up, g.limit)) { ok = false; break; }
                        if (lane == 0) {
                            // armed here and not with the other: the first states of a segment need no c, so that the
                            // chunk that was here before may have been waiting for its own until now
                            bar_expect(full_c + 8 * st, panels_v * kPanel);
                            for (int i = 0; i < panels_v; i++)
                                copy_box(stage + (2 * panels_k + i) * kPanel, &maps.c[pass], full_c + 8 * st, k.head * p.vd + i * 64,
                                         (int)row);
                        }
                        __syncwarp();
                        continue;
                    }
                    load_any(p.c_wide, stage + 2 * panels_k * kPanel, (const char*)p.c + (row * p.c_ld + (int64_t)k.head * p.vd) * 2,
                             p.c_ld * 2, p.vd, n);
                    load_any(p.b_wide, stage + panels_k * kPanel, (const char*)p.b + (row * p.b_ld + (int64_t)k.head * p.kd) * 2,
                             p.b_ld * 2, p.kd, n);
                    if (g.full)
                        load_any(p.a_wide, stage, (const char*)p.a + (row * p.a_ld + (int64_t)k.head * p.kd) * 2, p.a_ld * 2, p.kd, n);
                    asm volatile("cp.async.wait_all;" ::: "memory");
                    proxy_fence();
                    __syncwarp();
                    if (lane == 0) bar_arrive(bar), bar_arrive(full_c + 8 * st);
                }
            }
            // all products have reported before the CTA ends
            for (uint32_t i = c > (uint32_t)g.stages ? c - g.stages : 0; i < c && ok; i++) {
                const uint32_t at = 8 * (i % g.stages), parity = (i / g.stages) & 1;
                ok = warp_wait(empty + at, parity, gave_up, g.limit) &&
                     (!g.full || (warp_wait(used + at, parity, gave_up, g.limit) &&
                                  warp_wait(entered_a + at, parity, gave_up, g.limit)));
            }
            if (!ok) {  // let the copies under way land before the CTA ends
                const unsigned long long until = now_ns() + 1000000ull;
                while (now_ns() < until) {
                }
            }
        } else {
            // ---- products: one warp issues those of out, one those of the state, each in its own order
            uint32_t pieces = 0;
            bool by_hand = false;
            const bool of_state = warp == kMultiplyState;
            for (int w = blockIdx.x; w < g.total && ok && (of_state || g.full); w += gridDim.x) {
                const Work k = work_of(g, w);
                const Pass& p = *k.p;
                const int panels_k = (p.kd + 63) / 64;
                const uint32_t keys = (p.kd + 15) / 16, values = (p.vd + 15) / 16;  // of 16
                constexpr uint32_t kBase = (1u << 4) | B::kFormat | (128u >> 4) << 24;
                const uint32_t score_desc = kBase | (128u >> 3) << 17, enter_desc = kBase | (values * 2) << 17,
                               out_desc = enter_desc | 1u << 16, add_desc = kBase | (keys * 2) << 17 | 1u << 16;
                const uint64_t z = smem_desc(z_base, 16, 1024);
                for (int chunk = 0; chunk < k.chunks && ok; chunk++, c++) {
                    const uint32_t st = c % g.stages, stage = ring + st * g.stage_bytes, b_tile = stage + panels_k * kPanel;
                    if (!warp_wait(full + 8 * st, (c / g.stages) & 1, gave_up, g.limit)) { ok = false; break; }
                    if (of_state) {
                        const uint64_t b_turned = smem_desc(b_tile, kPanel, 1024);
                        if (c > 0 && !warp_wait(add_free, (c - 1) & 1, gave_up, g.limit)) { ok = false; break; }
#pragma unroll 1
                        for (int q = 0; q < kPieces && ok; q++, pieces++) {
                            const uint32_t slot = pieces % kSlots;
                            if (!warp_wait(c_ready + 8 * slot, (pieces / kSlots) & 1, gave_up, g.limit)) { ok = false; break; }
                            fence_after();
                            if (elect_one()) {
                                // small parts first: less of them is cut off
#pragma unroll
                                for (int part = kParts - 1; part >= 0; part--)
#pragma unroll
                                    for (int i = 0; i < kPiece / 16; i++)
                                        mma_ts(tmem + kColAdd, tmem + kColC + slot * kSlotCols + part * (kPiece / 2) + i * 8,
                                               b_turned + (q * (kPiece / 16) + i) * (2048 >> 4), add_desc,
                                               q > 0 || part < kParts - 1 || i > 0);
                                mma_done(c_free + 8 * slot);
                                if (q == kPieces - 1) {
                                    if (!g.withhold) mma_done(added);
                                    mma_done((g.full ? used : empty) + 8 * st);
                                }
                            }
                            __syncwarp();
                        }
                        continue;
                    }
                    const int n = tokens_of(k, chunk);
                    const uint64_t a = smem_desc(stage, 16, 1024), b = smem_desc(b_tile, 16, 1024),
                                   c_turned = smem_desc(stage + 2 * panels_k * kPanel, kPanel, 1024);
                    // the weights of the chunk before, in the place of the scores, are used up
                    if (c > 0 && !warp_wait(done, (c - 1) & 1, gave_up, g.limit)) { ok = false; break; }
                    if (by_hand && !warp_wait(out_free, (c - 1) & 1, gave_up, g.limit)) { ok = false; break; }
                    fence_after();
                    if (elect_one()) {
#pragma unroll 1
                        for (uint32_t i = 0; i < keys; i++)
                            mma_ss(tmem + kColScore, a + (i >> 2) * (kPanel >> 4) + (i & 3) * 2, b + (i >> 2) * (kPanel >> 4) + (i & 3) * 2,
                                   score_desc, i > 0);
                        mma_done(scored);
                    }
                    __syncwarp();
                    if (c > 0 && !warp_wait(out_free, (c - 1) & 1, gave_up, g.limit)) { ok = false; break; }
                    if (!warp_wait(z_ready, c & 1, gave_up, g.limit)) { ok = false; break; }
                    fence_after();
                    if (elect_one()) {
#pragma unroll 1
                        for (uint32_t i = 0; i < keys; i++)
                            mma_ss(tmem + kColOut, a + (i >> 2) * (kPanel >> 4) + (i & 3) * 2, z + (i >> 2) * (kPanel >> 4) + (i & 3) * 2,
                                   enter_desc, i > 0);
                        mma_done(entered);
                        mma_done(entered_a + 8 * st);
                    }
                    __syncwarp();
                    if (!warp_wait(weighted, c & 1, gave_up, g.limit)) { ok = false; break; }
                    fence_after();
                    by_hand = *(volatile uint32_t*)&tab.bad[c & 1] == c + 1;
                    if (elect_one()) {
                        if (!by_hand) {
#pragma unroll 1
                            for (int i = 0; i < (n + 15) / 16; i++)
                                mma_ts(tmem + kColOut, tmem + kColScore + i * 8, c_turned + i * (2048 >> 4), out_desc, true);
                        }
                        mma_done(done);
                    }
                    __syncwarp();
                }
            }
            for (uint32_t i = pieces > kSlots ? pieces - kSlots : 0; i < pieces && ok; i++)
                ok = warp_wait(c_free + 8 * (i % kSlots), (i / kSlots) & 1, gave_up, g.limit);
            if (!ok) {  // let the products under way end before the CTA does
                const unsigned long long until = now_ns() + 1000000ull;
                while (now_ns() < until) {
                }
            }
        }
    }
    __syncthreads();
    if (threadIdx.x == 0 && *gave_up) *g.status = 2;
    if (warp == kMultiply) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
}

// ---- 32-bit types -------------------------------------------------------------------------------

// The same passes in plain 32-bit arithmetic, in chunks of 32 tokens; a CTA a segment and head.  Z lies in registers, four
// keys x four values a thread (of every 64 x 64), and in shared memory, where the products with a read it; the next chunk's
// copies fly while one is worked on.  Shared memory is the bound: a warp's 32 multiply-adds of out take 10 of its cycles.
constexpr int kPlainChunk = 32, kPlainThreads = 256;
__host__ __device__ constexpr int plain_pitch(int d) { return (d + 3) / 4 * 4 + 4; }
constexpr int kWeightPitch = kPlainChunk + 4;
__host__ __device__ constexpr size_t plain_stage(int kd, int vd) { return (size_t)kPlainChunk * (2 * plain_pitch(kd) + plain_pitch(vd)); }
__host__ __device__ constexpr size_t plain_smem(int kd, int vd) {
    return sizeof(float) * (2 * plain_stage(kd, vd) + kPlainChunk * kWeightPitch + 2 * kPlainChunk + (size_t)(kd + 3) / 4 * 4 * plain_pitch(vd));
}
__device__ __forceinline__ void load_plain(float* dst, const float* src, int64_t pitch, int width, bool wide, int n) {
    const int p = plain_pitch(width), quads = (width + 3) / 4;
    for (int i = threadIdx.x; i < kPlainChunk * quads; i += kPlainThreads) {
        const int row = i / quads, col = (i - row * quads) * 4;
        const float* from = src + row * pitch + col;
        const uint32_t to = smem_u32(dst + row * p + col);
        if (wide) {
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(row < n ? from : src), "r"(row < n ? 16 : 0)
                         : "memory");
        } else {
#pragma unroll
            for (int k = 0; k < 4; k++) {
                const bool in = row < n && col + k < width;
                asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to + 4 * k), "l"(in ? from + k : src),
                             "r"(in ? 4 : 0)
                             : "memory");
            }
        }
    }
}
__device__ __forceinline__ float4 fma4(float a, float4 b, float4 c) {
    return make_float4(fmaf(a, b.x, c.x), fmaf(a, b.y, c.y), fmaf(a, b.z, c.z), fmaf(a, b.w, c.w));
}
__device__ __forceinline__ float dot4(float4 a, float4 b, float c) {
    return fmaf(a.x, b.x, fmaf(a.y, b.y, fmaf(a.z, b.z, fmaf(a.w, b.w, c))));
}
__device__ __forceinline__ const float4& quad(const float* p) { return *reinterpret_cast<const float4*>(p); }
// kTiles: tiles of 64 that the larger of keys and values takes.
template <int kTiles>
__global__ void __launch_bounds__(kPlainThreads, kTiles == 1 ? 2 : 1) attention_plain_kernel(const __grid_constant__ Args g) {
    extern __shared__ __align__(16) float sm[];
    pdl_wait();
    pdl_trigger();
    const Work k = work_of(g, blockIdx.x);
    const Pass& p = *k.p;
    const int kd = p.kd, vd = p.vd, kd4 = (kd + 3) / 4 * 4, vd4 = (vd + 3) / 4 * 4, kp = plain_pitch(kd), vp = plain_pitch(vd);
    const int stage = (int)plain_stage(kd, vd);
    float* const weights = sm + 2 * stage;
    float* const powers = weights + kPlainChunk * kWeightPitch;  // d^0 .. d^31
    float* const left = powers + kPlainChunk;
    float* const zs = left + kPlainChunk;                         // [kd4][vp]
    const int t = threadIdx.x, tx = t & 15, ty = t >> 4;
    const int64_t way = p.reverse ? -1 : 1;
    const int64_t row0 = p.reverse ? k.s.row0 + k.s.len - 1 : k.s.row0;
    const bool full = g.full;
    auto fetch = [&](int chunk) {
        const int at = chunk * kPlainChunk, n = min(kPlainChunk, k.s.len - at);
        const int64_t row = row0 + way * at;
        float* const to = sm + (chunk & 1) * stage;
        if (full) load_plain(to, (const float*)p.a + row * p.a_ld + (int64_t)k.head * kd, way * p.a_ld, kd, p.a_wide == 16, n);
        load_plain(to + kPlainChunk * kp, (const float*)p.b + row * p.b_ld + (int64_t)k.head * kd, way * p.b_ld, kd, p.b_wide == 16, n);
        load_plain(to + 2 * kPlainChunk * kp, (const float*)p.c + row * p.c_ld + (int64_t)k.head * vd, way * p.c_ld, vd, p.c_wide == 16, n);
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    const int chunks = (k.s.len + kPlainChunk - 1) / kPlainChunk;
    if (chunks) fetch(0);
    if (t < kPlainChunk) powers[t] = exp2f(k.l2 * t);
    const float* from = state_in(g, k);
    float4 z[kTiles][kTiles][4];
#pragma unroll
    for (int a = 0; a < kTiles; a++)
#pragma unroll
        for (int b = 0; b < kTiles; b++)
#pragma unroll
            for (int y = 0; y < 4; y++) {
                const int key = a * 64 + ty * 4 + y, value = b * 64 + tx * 4;
                float v[4];
#pragma unroll
                for (int x = 0; x < 4; x++)
                    v[x] = from && key < kd && value + x < vd ? from[(int64_t)key * p.k_step + (int64_t)(value + x) * p.v_step] : 0.0f;
                z[a][b][y] = make_float4(v[0], v[1], v[2], v[3]);
            }
    for (int chunk = 0; chunk < chunks; chunk++) {
        const int at = chunk * kPlainChunk, n = min(kPlainChunk, k.s.len - at);
        if (chunk + 1 < chunks) {
            fetch(chunk + 1);
            asm volatile("cp.async.wait_group 1;" ::: "memory");
        } else {
            asm volatile("cp.async.wait_group 0;" ::: "memory");
        }
        if (full) {
#pragma unroll
            for (int a = 0; a < kTiles; a++)
#pragma unroll
                for (int b = 0; b < kTiles; b++)
#pragma unroll
                    for (int y = 0; y < 4; y++) {
                        const int key = a * 64 + ty * 4 + y, value = b * 64 + tx * 4;
                        if (key < kd4 && value < vd4) *reinterpret_cast<float4*>(zs + key * vp + value) = z[a][b][y];
                    }
        }
        if (t < kPlainChunk) left[t] = t < n ? p.gain * exp2f(k.l2 * (n - p.e - t)) : 0.0f;
        __syncthreads();
        const float *const as = sm + (chunk & 1) * stage, *const bs = as + kPlainChunk * kp, *const cs = bs + kPlainChunk * kp;
        if (full) {
            // weights: two tokens of a and two of c a thread
            float s[2][2] = {{0.0f, 0.0f}, {0.0f, 0.0f}};
            for (int x = 0; x < kd4; x += 4) {
                const float4 a0 = quad(as + ty * 2 * kp + x), a1 = quad(as + (ty * 2 + 1) * kp + x);
                const float4 b0 = quad(bs + tx * kp + x), b1 = quad(bs + (tx + 16) * kp + x);
                s[0][0] = dot4(a0, b0, s[0][0]), s[0][1] = dot4(a0, b1, s[0][1]);
                s[1][0] = dot4(a1, b0, s[1][0]), s[1][1] = dot4(a1, b1, s[1][1]);
            }
#pragma unroll
            for (int y = 0; y < 2; y++)
#pragma unroll
                for (int x = 0; x < 2; x++) {
                    const int i = ty * 2 + y, j = tx + 16 * x;
                    weights[i * kWeightPitch + j] = j <= i ? s[y][x] * (p.intra * powers[i - j]) : 0.0f;
                }
            // a token after a row's own weighs nothing, whatever it holds: infinities and NaN are kept out of the sums
            bool odd = false;
            for (int v0 = tx * 4; v0 < vd4; v0 += 64)
#pragma unroll
                for (int y = 0; y < 2; y++) {
                    const float4 c = quad(cs + (ty * 2 + y) * vp + v0);
                    odd |= !(fabsf(c.x) < INFINITY && fabsf(c.y) < INFINITY && fabsf(c.z) < INFINITY && fabsf(c.w) < INFINITY);
                }
            odd = __syncthreads_or(odd);
            // out: two tokens and four values a thread
            for (int v0 = tx * 4; v0 < vd4; v0 += 64) {
                float4 o[2] = {make_float4(0.0f, 0.0f, 0.0f, 0.0f), make_float4(0.0f, 0.0f, 0.0f, 0.0f)};
                auto step = [&](const float* rows, int pitch, const float* columns, int x) {
                    const float4 u0 = quad(rows + x), u1 = quad(rows + pitch + x);
                    const float4 c0 = quad(columns + x * vp), c1 = quad(columns + (x + 1) * vp), c2 = quad(columns + (x + 2) * vp),
                                 c3 = quad(columns + (x + 3) * vp);
                    o[0] = fma4(u0.x, c0, fma4(u0.y, c1, fma4(u0.z, c2, fma4(u0.w, c3, o[0]))));
                    o[1] = fma4(u1.x, c0, fma4(u1.y, c1, fma4(u1.z, c2, fma4(u1.w, c3, o[1]))));
                };
#pragma unroll 2
                for (int x = 0; x < kd4; x += 4) step(as + ty * 2 * kp, kp, zs + v0, x);
#pragma unroll
                for (int y = 0; y < 2; y++) {
                    const float f = p.inter * exp2f(k.l2 * (ty * 2 + y + p.e));
                    o[y] = make_float4(o[y].x * f, o[y].y * f, o[y].z * f, o[y].w * f);
                }
                if (!odd) {
#pragma unroll 2
                    for (int x = 0; x < ty * 2 + 2; x += 4) step(weights + ty * 2 * kWeightPitch, kWeightPitch, cs + v0, x);
                } else {
#pragma unroll
                    for (int y = 0; y < 2; y++)
                        for (int j = 0; j <= ty * 2 + y; j++)
                            o[y] = fma4(weights[(ty * 2 + y) * kWeightPitch + j], quad(cs + j * vp + v0), o[y]);
                }
#pragma unroll
                for (int y = 0; y < 2; y++) {
                    const int i = ty * 2 + y;
                    if (i >= n) continue;
                    float* to = (float*)p.out + (row0 + way * (at + i)) * p.out_ld + (int64_t)k.head * vd + v0;
                    if (p.out_wide == 16) {
                        *reinterpret_cast<float4*>(to) = o[y];
                    } else {
                        to[0] = o[y].x;
                        if (v0 + 1 < vd) to[1] = o[y].y;
                        if (v0 + 2 < vd) to[2] = o[y].z;
                        if (v0 + 3 < vd) to[3] = o[y].w;
                    }
                }
            }
        }
        // Z
        const float decay = exp2f(k.l2 * n);
#pragma unroll
        for (int a = 0; a < kTiles; a++)
#pragma unroll
            for (int b = 0; b < kTiles; b++) {
                const int key = a * 64 + ty * 4, value = b * 64 + tx * 4;
                if (key >= kd4 || value >= vd4) continue;
                float4 add[4];
#pragma unroll
                for (int y = 0; y < 4; y++) add[y] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
                for (int j = 0; j < n; j++) {
                    const float4 u = quad(bs + j * kp + key), v = quad(cs + j * vp + value);
                    const float w = left[j];
                    const float4 vw = make_float4(v.x * w, v.y * w, v.z * w, v.w * w);
                    add[0] = fma4(u.x, vw, add[0]), add[1] = fma4(u.y, vw, add[1]);
                    add[2] = fma4(u.z, vw, add[2]), add[3] = fma4(u.w, vw, add[3]);
                }
#pragma unroll
                for (int y = 0; y < 4; y++) z[a][b][y] = fma4(decay, z[a][b][y], add[y]);
            }
        __syncthreads();
    }
    float* const to = state_out(g, k);
    if (to) {
#pragma unroll
        for (int a = 0; a < kTiles; a++)
#pragma unroll
            for (int b = 0; b < kTiles; b++)
#pragma unroll
                for (int y = 0; y < 4; y++) {
                    const int key = a * 64 + ty * 4 + y, value = b * 64 + tx * 4;
                    const float v[4] = {z[a][b][y].x, z[a][b][y].y, z[a][b][y].z, z[a][b][y].w};
#pragma unroll
                    for (int x = 0; x < 4; x++)
                        if (key < kd && value + x < vd) to[(int64_t)key * p.k_step + (int64_t)(value + x) * p.v_step] = v[x];
                }
    }
    if (t == 0) decay_out(k, g.log_decay);
}

// ---- along the segments, along the ranks, single tokens -----------------------------------------

struct FoldArgs {
    float* states[2];          // [slots][heads][size]: what each segment adds; on return the state that enters it
    const float* first[2];     // [sequences][heads][size], null: zero
    float* summary[2];         // null: not wanted; else the last segments' additions are there too
    int reverse[2];
    const Segment* segments;   // by slot: those of a sequence in the order of time
    const int32_t* begin;      // [sequences that are cut + 1]
    const float* log_decay;
    int heads, size;
};
__global__ void __launch_bounds__(256) attention_fold_kernel(const __grid_constant__ FoldArgs g) {
    pdl_wait();
    pdl_trigger();
    const int which = blockIdx.z, cut = blockIdx.x / g.heads, h = blockIdx.x - cut * g.heads;
    const int at = blockIdx.y * 256 + threadIdx.x;
    const int lo = g.begin[cut], n = g.begin[cut + 1] - lo;
    const int64_t s = g.segments[lo].seq;
    const float l2 = log2_decay(g.log_decay, h);
    const int64_t unit = (int64_t)g.heads * g.size;
    if (at < g.size) {
        float z = g.first[which] ? g.first[which][s * unit + (int64_t)h * g.size + at] : 0.0f;
        float* const states = g.states[which] + (int64_t)h * g.size + at;
        // a batch is read before any of it is written: the trips to memory do not wait for one another
        constexpr int kBatch = 8;
        for (int i0 = 0; i0 < n; i0 += kBatch) {
            float here[kBatch], decay[kBatch];
#pragma unroll
            for (int y = 0; y < kBatch; y++) {
                const int i = i0 + y, id = g.reverse[which] ? lo + n - 1 - i : lo + i;
                here[y] = i + 1 < n || (i < n && g.summary[which]) ? states[id * unit] : 0.0f;
                decay[y] = i < n ? exp2f(l2 * (float)g.segments[id].len) : 0.0f;
            }
#pragma unroll
            for (int y = 0; y < kBatch; y++) {
                const int i = i0 + y, id = g.reverse[which] ? lo + n - 1 - i : lo + i;
                if (i >= n) break;
                states[id * unit] = z;
                z = fmaf(decay[y], z, here[y]);
            }
        }
        if (g.summary[which])
            g.summary[which][s * (unit + g.heads) + g.heads + (int64_t)h * g.size + at] = z;
    }
    if (g.summary[which] && at == 0) {
        const int64_t len = g.segments[lo].seq_len;
        g.summary[which][s * (unit + g.heads) + h] = len ? (float)exp((double)g.log_decay[h] * (double)len) : 1.0f;
    }
}

__global__ void __launch_bounds__(256) attention_join_kernel(int P, int first_rank, int heads, int size,
                                                             const float* __restrict__ gathered,
                                                             const float* __restrict__ first, float* __restrict__ out,
                                                             int reverse) {
    pdl_wait();
    pdl_trigger();
    const int h = blockIdx.y, at = blockIdx.x * 256 + threadIdx.x;
    if (at >= size) return;
    const int64_t block = (int64_t)heads * (1 + size), state = (int64_t)h * size + at;
    const float* const blocks = gathered + (int64_t)blockIdx.z * P * block;
    const int r = first_rank + blockIdx.z, n = reverse ? P - 1 - r : r;
    float z = first ? first[state] : 0.0f;
#pragma unroll 4
    for (int i = 0; i < n; i++) {
        const float* const from = blocks + (reverse ? P - 1 - i : i) * block;
        z = fmaf(from[h], z, from[heads + state]);
    }
    out[(int64_t)blockIdx.z * heads * size + state] = z;
}

// One token of one head (blockIdx.x = row * heads + head), a slice of its values: a state is read and written once.
// kWide: four values a thread.
template <typename T, bool kWide>
__global__ void __launch_bounds__(256) attention_step_kernel(int heads, int kd, int vd, int slice, float scale,
                                                             const T* __restrict__ q, int64_t q_ld, const T* __restrict__ k,
                                                             int64_t k_ld, const T* __restrict__ v, int64_t v_ld,
                                                             const float* __restrict__ log_decay,
                                                             const int32_t* __restrict__ slots, int64_t n_slots,
                                                             const float* state_in, float* state_out, T* __restrict__ o,
                                                             int64_t o_ld) {
    constexpr int V = kWide ? 4 : 1;
    __shared__ float qs[kMostSize], ks[kMostSize];
    __shared__ __align__(16) float sums[256 * V];
    pdl_wait();
    pdl_trigger();
    const int64_t row = blockIdx.x / heads;
    const int h = (int)(blockIdx.x - row * heads), t = threadIdx.x;
    const int64_t slot = slots ? slots[row] : row;
    const int v0 = blockIdx.y * slice, width = min(slice, vd - v0), across = (width + V - 1) / V;
    T* const to = o + row * o_ld + (int64_t)h * vd + v0;
    if (slot < 0 || slot >= n_slots) {
        for (int i = t; i < width; i += 256) to[i] = from_float<T>(0.0f);
        return;
    }
    for (int i = t; i < kd; i += 256) {
        qs[i] = scale * to_float(q[row * q_ld + (int64_t)h * kd + i]);
        ks[i] = to_float(k[row * k_ld + (int64_t)h * kd + i]);
    }
    const float decay = exp2f(log2_decay(log_decay, h));
    const int groups = 256 / across, group = t / across, col = (t - group * across) * V;
    float vs[V], sum[V];
#pragma unroll
    for (int i = 0; i < V; i++) {
        vs[i] = group < groups && col + i < width ? to_float(v[row * v_ld + (int64_t)h * vd + v0 + col + i]) : 0.0f;
        sum[i] = 0.0f;
    }
    __syncthreads();
    const int64_t base = (slot * heads + h) * (int64_t)kd * vd + v0 + col;
    if (group < groups) {
        // the tables may be one: all of a batch is read before any of it is written
        constexpr int kBatch = 8;
        for (int key0 = group; key0 < kd; key0 += groups * kBatch) {
            Pack<float, V> s[kBatch];
#pragma unroll
            for (int y = 0; y < kBatch; y++)
                if (key0 + y * groups < kd)
                    s[y] = *reinterpret_cast<const Pack<float, V>*>(state_in + base + (int64_t)(key0 + y * groups) * vd);
#pragma unroll
            for (int y = 0; y < kBatch; y++) {
                const int key = key0 + y * groups;
                if (key >= kd) break;
#pragma unroll
                for (int i = 0; i < V; i++) {
                    s[y].v[i] = fmaf(decay, s[y].v[i], ks[key] * vs[i]);
                    sum[i] = fmaf(qs[key], s[y].v[i], sum[i]);
                }
                *reinterpret_cast<Pack<float, V>*>(state_out + base + (int64_t)key * vd) = s[y];
            }
        }
    }
#pragma unroll
    for (int i = 0; i < V; i++) sums[t * V + i] = sum[i];
    __syncthreads();
    for (int i = t; i < width; i += 256) {
        float all = 0.0f;
        for (int y = 0; y < groups; y++) all += sums[(y * across) * V + i];
        to[i] = from_float<T>(all);
    }
}

}  // namespace

struct sparbit_linear_attention_plan_s {
    int n_seqs = 0, heads = 0, kd = 0, vd = 0, dtype = 0;
    float scale = 1.0f;
    size_t rows = 0;
    std::vector<Segment> slots, list;  // segments of the sequences that are cut, by slot; all, the longest first
    std::vector<int32_t> begin;        // slots of each sequence that is cut
    char* work = nullptr;
    int device = -1, sm_count = 0;
    unsigned long long limit = kWaitNs;
    int withhold = 0;
    void* encode = nullptr;            // cuTensorMapEncodeTiled

    bool split() const { return !slots.empty(); }
    size_t states() const { return (size_t)heads * kd * vd; }
    size_t block() const { return states() + heads; }
    size_t off_slots() const { return 256; }
    size_t off_list() const { return off_slots() + round_up(slots.size() * sizeof(Segment), 256); }
    size_t off_begin() const { return off_list() + round_up(list.size() * sizeof(Segment), 256); }
    size_t off_states(int which) const {
        return off_begin() + round_up(begin.size() * sizeof(int32_t), 256) +
               which * round_up(slots.size() * states() * sizeof(float), 256);
    }
    size_t work_bytes() const { return off_states(2); }
};

namespace {

using Plan = sparbit_linear_attention_plan_s;

int ready(const Plan* p) {
    if (!p->work) return SPARBIT_ERR_WORKSPACE;
    int cur = -1;
    CU(cudaGetDevice(&cur));
    return cur == p->device ? SPARBIT_OK : SPARBIT_ERR_ARG;
}

// A tensor of rows of heads x size elements.
struct Rows {
    const void* p;
    size_t ld;
    int size;
};

int alignment(const Plan* p, const Rows& r) {
    const size_t es = elem_size(p->dtype);
    return common_alignment((uintptr_t)r.p | r.ld * es | r.size * es, 16);
}

Pass make_pass(const Plan* p, const Rows& a, const Rows& b, const Rows& c, const Rows& out, bool reverse) {
    Pass x = {};
    x.a = a.p, x.b = b.p, x.c = c.p, x.out = (void*)out.p;
    x.a_ld = (int64_t)a.ld, x.b_ld = (int64_t)b.ld, x.c_ld = (int64_t)c.ld, x.out_ld = (int64_t)out.ld;
    x.kd = b.size, x.vd = c.size;
    x.a_wide = alignment(p, a), x.b_wide = alignment(p, b), x.c_wide = alignment(p, c), x.out_wide = alignment(p, out);
    x.reverse = reverse, x.e = reverse ? 0 : 1;
    x.inter = reverse ? 1.0f : p->scale, x.intra = p->scale, x.gain = reverse ? p->scale : 1.0f;
    x.unit_in = x.unit_out = (int64_t)p->states();
    x.k_step = c.size, x.v_step = 1;
    return x;
}
// The state of this pass lies as [values][keys].
void turned(Pass& x) { x.k_step = 1, x.v_step = x.kd; }

Args common_args(const Plan* p) {
    Args g = {};
    g.list = (const Segment*)(p->work + p->off_list());
    g.heads = p->heads;
    g.status = (uint32_t*)p->work;
    g.limit = p->limit;
    g.withhold = p->withhold;
    return g;
}

typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                             const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                             CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// One head's size must be a multiple of the products' 16 elements: a box past it brings the next head's.
bool encode(const Plan* p, CUtensorMap* map, const void* q, int64_t ld, int size, int box_rows = kChunk, int box_width = 64) {
    const cuuint64_t dims[2] = {(cuuint64_t)p->heads * size, (cuuint64_t)p->rows}, strides[1] = {(cuuint64_t)ld * 2};
    const cuuint32_t box[2] = {(cuuint32_t)box_width, (cuuint32_t)box_rows}, one[2] = {1, 1};
    return ((EncodeFn)p->encode)(map, p->dtype == SPARBIT_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
                                 2, const_cast<void*>(q), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                 box_width == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                                 CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                 CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int run(const Plan* p, Args& g, cudaStream_t st) {
    g.total = (int)p->list.size() * p->heads * g.n_passes;
    if (p->dtype == SPARBIT_F32) {
        size_t smem = 0;
        for (int i = 0; i < g.n_passes; i++) smem = std::max(smem, plain_smem(g.pass[i].kd, g.pass[i].vd));
        // what a function is allowed is the function's and not this plan's: the same whatever the plan, since another thread
        // may be setting it for its own
        auto launch_it = [&](auto kernel, int most) {
            CU(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)plain_smem(most, most)));
            CU(launch(kernel, dim3(g.total), dim3(kPlainThreads), smem, st, g));
            return (int)SPARBIT_OK;
        };
        return std::max(p->kd, p->vd) <= 64 ? launch_it(attention_plain_kernel<1>, 64)
                                            : launch_it(attention_plain_kernel<2>, kMostSize);
    }
    uint32_t state = 0;
    g.stage_bytes = 0;
    for (int i = 0; i < g.n_passes; i++) {
        const uint32_t pk = (g.pass[i].kd + 63) / 64, pv = (g.pass[i].vd + 63) / 64;
        g.stage_bytes = std::max(g.stage_bytes, (2 * pk + pv) * kPanel);
        state = std::max(state, pk * kPanel);
    }
    g.stages = (int)std::min<uint32_t>(kMostStages, (kRing - state) / g.stage_bytes);
    g.early = g.full;
    for (int i = 0; i < g.n_passes; i++) {
        const Pass &x = g.pass[i], &y = g.pass[0];
        g.early = g.early && (x.kd + 63) / 64 == (y.kd + 63) / 64 && (x.vd + 63) / 64 == (y.vd + 63) / 64;
    }
    const size_t smem = kTensorSmem;
    Maps maps;
    for (int i = 0; i < g.n_passes; i++) {
        Pass& x = g.pass[i];
        x.tiled = x.b_wide == 16 && x.c_wide == 16 && (!g.full || x.a_wide == 16) && x.kd % 16 == 0 && x.vd % 16 == 0 &&
                  p->rows >= kChunk && p->rows <= 0x7fffffffu && encode(p, &maps.b[i], x.b, x.b_ld, x.kd) &&
                  encode(p, &maps.c[i], x.c, x.c_ld, x.vd) && (!g.full || encode(p, &maps.a[i], x.a, x.a_ld, x.kd));
        // 64 values a warp of 128, 32 of 64 or 32
        x.out_tiled = g.full && x.out_wide == 16 && (x.vd == 32 || x.vd == 64 || x.vd == 128) && p->rows >= 32 &&
                      p->rows <= 0x7fffffffu && encode(p, &maps.out[i], x.out, x.out_ld, x.vd, 32, x.vd == 128 ? 64 : 32);
    }
    const dim3 grid(std::min(g.total, p->sm_count));
    auto launch_it = [&](auto kernel) {
        CU(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
        CU(launch(kernel, grid, dim3(kTensorThreads), smem, st, g, maps));
        return (int)SPARBIT_OK;
    };
    return p->dtype == SPARBIT_BF16 ? launch_it(attention_tensor_kernel<__nv_bfloat16>) : launch_it(attention_tensor_kernel<__half>);
}

int fold(const Plan* p, FoldArgs& f, int n, const float* log_decay, cudaStream_t st) {
    f.segments = (const Segment*)(p->work + p->off_slots());
    f.begin = (const int32_t*)(p->work + p->off_begin());
    f.log_decay = log_decay;
    f.heads = p->heads, f.size = p->kd * p->vd;
    for (int i = 0; i < n; i++) f.states[i] = (float*)(p->work + p->off_states(i));
    CU(launch(attention_fold_kernel, dim3((unsigned)((p->begin.size() - 1) * p->heads), (unsigned)((f.size + 255) / 256), (unsigned)n),
              dim3(256), 0, st, f));
    return SPARBIT_OK;
}

// What each segment adds to a state of its direction, for fold; `all`: the last ones of a sequence too, and with them the
// states of the sequences that are whole.
void local_states(const Plan* p, Pass& x, int which, bool all) {
    x.out = nullptr;
    x.slots_out = (float*)(p->work + p->off_states(which));
    x.skip_ends = !all;
}
void from_segment(const Plan* p, Pass& x, int which) {
    if (p->split()) x.slots_in = (const float*)(p->work + p->off_states(which));
}
void into_summary(const Plan* p, Pass& x, float* summary) {
    if (!summary) return;
    x.z_out = summary + p->heads;
    x.decay_out = summary;
    x.unit_out = (int64_t)p->block();
}

bool bad_rows(const Plan* p, const Rows& r) { return bad_pitch(r.ld, (size_t)p->heads * r.size, p->rows); }
Region region(const Plan* p, const Rows& r) {
    const size_t es = elem_size(p->dtype);
    return Region{r.p, p->rows, (size_t)p->heads * r.size * es, r.ld * es};
}
int overlaps(const Region* ins, int n, const Region* outs, int m) {
    for (int i = 0; i < m; i++) {
        for (int j = 0; j < n; j++)
            if (regions_overlap(outs[i], ins[j])) return SPARBIT_ERR_ALIAS;
        for (int j = 0; j < i; j++)
            if (regions_overlap(outs[i], outs[j])) return SPARBIT_ERR_ALIAS;
    }
    return SPARBIT_OK;
}

// Tokens that segments are multiples of.
int unit_of(int dtype) { return dtype == SPARBIT_F32 ? kPlainChunk : kChunk; }

// Units of a segment, at most; chosen for the least estimated time, in units' times: a launch takes what the SM with the
// most of them has, and about one more for each segment; the launch that leaves the states about two thirds of the main
// one; the fold between them about two.
int64_t segment_units(const std::vector<int64_t>& units, int heads, int slots) {
    int64_t longest = 1;
    for (int64_t c : units) longest = std::max(longest, c);
    int64_t best = longest;
    double least = 1e300;
    for (int64_t len = longest;; len = std::min(len - 1, (len * 7 + 7) / 8)) {
        if (len < 1) break;
        double items = 0, all = 0;
        for (int64_t c : units) items += (double)((c + len - 1) / len), all += (double)c;
        items *= heads, all *= heads;
        const double rounds = items <= 3 * slots ? ceil(items / slots) * (len + 1) : (all + items) / slots + len * 0.5;
        const double cost = len < longest ? 1.67 * rounds + 2 : rounds;
        if (cost < least) least = cost, best = len;
    }
    return best;
}

}  // namespace

extern "C" {

int sparbit_linear_attention_plan_create(int n_seqs, const size_t* lengths, int heads, int key_size, int value_size,
                                         int dtype, float scale, sparbit_linear_attention_plan_t** out) {
    if (!out) return SPARBIT_ERR_ARG;
    *out = nullptr;
    if (!lengths || n_seqs < 1 || heads < 1 || key_size < 1 || value_size < 1 || !known_dtype(dtype) || !isfinite(scale))
        return SPARBIT_ERR_ARG;
    if (key_size > SPARBIT_LINEAR_ATTENTION_MAX_SIZE || value_size > SPARBIT_LINEAR_ATTENTION_MAX_SIZE || heads > 4096 ||
        n_seqs > 65535)
        return SPARBIT_ERR_LIMIT;
    const size_t most = kMostElements / ((size_t)heads * std::max(key_size, value_size));
    size_t rows = 0;
    for (int s = 0; s < n_seqs; s++) {
        if (lengths[s] > most - rows) return SPARBIT_ERR_OVERFLOW;
        rows += lengths[s];
        if (lengths[s] > 0x7fffffffu) return SPARBIT_ERR_LIMIT;
    }
    Plan* p = new (std::nothrow) Plan();
    if (!p) return SPARBIT_ERR_NOMEM;
    try {
        p->n_seqs = n_seqs, p->heads = heads, p->kd = key_size, p->vd = value_size, p->dtype = dtype;
        p->scale = scale, p->rows = rows;
        const int64_t unit = unit_of(dtype);
        std::vector<int64_t> units;
        for (int s = 0; s < n_seqs; s++) units.push_back(((int64_t)lengths[s] + unit - 1) / unit);
        // CTAs of 32-bit heads up to 64 come two to an SM
        const int64_t len = segment_units(units, heads, dtype == SPARBIT_F32 && std::max(key_size, value_size) <= 64 ? 2 * kSms : kSms);
        int64_t row = 0;
        for (int s = 0; s < n_seqs; s++) {
            const int64_t n = std::max<int64_t>(1, (units[s] + len - 1) / len), each = (units[s] + n - 1) / n * unit;
            if (n > 1) p->begin.push_back((int32_t)p->slots.size());
            int64_t at = 0;
            do {
                const int64_t left = (int64_t)lengths[s] - at, here = std::min(each, left);
                const int32_t slot = n > 1 ? (int32_t)p->slots.size() : -1;
                p->list.push_back(Segment{row + at, (int64_t)lengths[s], (int32_t)here, s, slot,
                                          (at == 0 ? 1 : 0) | (here == left ? 2 : 0)});
                if (slot >= 0) p->slots.push_back(p->list.back());
                at += here;
            } while (at < (int64_t)lengths[s]);
            row += (int64_t)lengths[s];
        }
        p->begin.push_back((int32_t)p->slots.size());
        if (p->list.size() > 0x7fffffffu / 3 / heads) {
            delete p;
            return SPARBIT_ERR_LIMIT;
        }
        std::stable_sort(p->list.begin(), p->list.end(), [](const Segment& a, const Segment& b) { return a.len > b.len; });
    } catch (const std::bad_alloc&) {
        delete p;
        return SPARBIT_ERR_NOMEM;
    }
    *out = p;
    return SPARBIT_OK;
}

int sparbit_linear_attention_plan_destroy(sparbit_linear_attention_plan_t* p) {
    delete p;
    return SPARBIT_OK;
}

size_t sparbit_linear_attention_plan_workspace_bytes(const sparbit_linear_attention_plan_t* p) {
    return p ? p->work_bytes() : 0;
}

int sparbit_linear_attention_plan_set_workspace(sparbit_linear_attention_plan_t* p, void* dev, size_t bytes) {
    if (!p) return SPARBIT_ERR_ARG;
    if (!dev || bytes < p->work_bytes() || (uintptr_t)dev % 16) return SPARBIT_ERR_WORKSPACE;
    p->work = nullptr;
    CU(cudaGetDevice(&p->device));
    CU(cudaDeviceGetAttribute(&p->sm_count, cudaDevAttrMultiProcessorCount, p->device));
    if (p->dtype != SPARBIT_F32) {
        cudaDriverEntryPointQueryResult found;
        CU(cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p->encode, 12000, cudaEnableDefault, &found));
        if (!p->encode || found != cudaDriverEntryPointSuccess)
            return record_cuda_error((int)cudaErrorNotSupported, "cuTensorMapEncodeTiled");
    }
    char* base = (char*)dev;
    CU(cudaMemset(base, 0, 256));
    if (p->split())
        CU(cudaMemcpy(base + p->off_slots(), p->slots.data(), p->slots.size() * sizeof(Segment), cudaMemcpyHostToDevice));
    CU(cudaMemcpy(base + p->off_list(), p->list.data(), p->list.size() * sizeof(Segment), cudaMemcpyHostToDevice));
    CU(cudaMemcpy(base + p->off_begin(), p->begin.data(), p->begin.size() * sizeof(int32_t), cudaMemcpyHostToDevice));
    CU(cudaDeviceSynchronize());
    p->work = base;
    return SPARBIT_OK;
}

int sparbit_linear_attention_forward(sparbit_linear_attention_plan_t* p, const void* q, size_t q_ld, const void* k,
                                     size_t k_ld, const void* v, size_t v_ld, const float* log_decay, const float* first,
                                     void* o, size_t o_ld, float* summary, void* stream) {
    if (!p) return SPARBIT_ERR_ARG;
    const Rows rq{o ? q : nullptr, q_ld, p->kd}, rk{k, k_ld, p->kd}, rv{v, v_ld, p->vd}, ro{o, o_ld, p->vd};
    if (!log_decay || (p->rows && (!k || !v || (o && !q)))) return SPARBIT_ERR_ARG;
    if (bad_rows(p, rk) || bad_rows(p, rv) || (o && (bad_rows(p, rq) || bad_rows(p, ro)))) return SPARBIT_ERR_ARG;
    const size_t states = p->n_seqs * p->states() * 4;
    const Region ins[] = {region(p, rq), region(p, rk), region(p, rv), {log_decay, 1, (size_t)p->heads * 4, 0},
                          {first, 1, states, 0}, {p->work, 1, p->work_bytes(), 0}};
    const Region outs[] = {region(p, ro), {summary, 1, p->n_seqs * p->block() * 4, 0}};
    int e = overlaps(ins, 6, outs, 2);
    if (e == SPARBIT_OK && (misaligned(elem_size(p->dtype), {rq.p, k, v, o}) || misaligned(4, {log_decay, first, summary})))
        e = SPARBIT_ERR_ARG;
    if (e == SPARBIT_OK) e = ready(p);
    if (e != SPARBIT_OK || (!o && !summary)) return e;
    const cudaStream_t st = (cudaStream_t)stream;
    const Pass main = make_pass(p, rq, rk, rv, ro, false);
    Args g = common_args(p);
    g.n_passes = 1;
    g.log_decay = log_decay;
    if (p->split()) {
        g.pass[0] = main;
        local_states(p, g.pass[0], 0, !o);
        FoldArgs f = {};
        f.first[0] = first;
        if (!o) {
            g.pass[0].z_in = first;
            into_summary(p, g.pass[0], summary);
            f.summary[0] = summary;
        }
        e = run(p, g, st);
        if (e == SPARBIT_OK) e = fold(p, f, 1, log_decay, st);
        if (e != SPARBIT_OK || !o) return e;
    }
    g.full = o != nullptr;
    g.pass[0] = main;
    g.pass[0].z_in = first;
    from_segment(p, g.pass[0], 0);
    into_summary(p, g.pass[0], summary);
    return run(p, g, st);
}

int sparbit_linear_attention_backward(sparbit_linear_attention_plan_t* p, const void* q, size_t q_ld, const void* k,
                                      size_t k_ld, const void* v, size_t v_ld, const float* log_decay, const float* first,
                                      const void* d_o, size_t do_ld, const float* dlast, void* dq, size_t dq_ld, void* dk,
                                      size_t dk_ld, void* dv, size_t dv_ld, float* dsummary, void* stream) {
    if (!p || !dq != !dk || !dq != !dv) return SPARBIT_ERR_ARG;
    const Rows rq{q, q_ld, p->kd}, rk{dq ? k : nullptr, k_ld, p->kd}, rv{dq ? v : nullptr, v_ld, p->vd},
        rd{d_o, do_ld, p->vd}, oq{dq, dq_ld, p->kd}, ok{dk, dk_ld, p->kd}, ov{dv, dv_ld, p->vd};
    if (!log_decay || (p->rows && (!q || !d_o || (dq && (!k || !v))))) return SPARBIT_ERR_ARG;
    if (bad_rows(p, rq) || bad_rows(p, rd)) return SPARBIT_ERR_ARG;
    if (dq && (bad_rows(p, rk) || bad_rows(p, rv) || bad_rows(p, oq) || bad_rows(p, ok) || bad_rows(p, ov)))
        return SPARBIT_ERR_ARG;
    const size_t states = p->n_seqs * p->states() * 4;
    const Region ins[] = {region(p, rq), region(p, rk), region(p, rv), region(p, rd), {log_decay, 1, (size_t)p->heads * 4, 0},
                          {dq ? first : nullptr, 1, states, 0}, {dlast, 1, states, 0}, {p->work, 1, p->work_bytes(), 0}};
    const Region outs[] = {region(p, oq), region(p, ok), region(p, ov), {dsummary, 1, p->n_seqs * p->block() * 4, 0}};
    int e = overlaps(ins, 8, outs, 4);
    if (e == SPARBIT_OK && (misaligned(elem_size(p->dtype), {q, rk.p, rv.p, d_o, dq, dk, dv}) ||
                            misaligned(4, {log_decay, dq ? first : nullptr, dlast, dsummary})))
        e = SPARBIT_ERR_ARG;
    if (e == SPARBIT_OK) e = ready(p);
    if (e != SPARBIT_OK || (!dq && !dsummary)) return e;
    const cudaStream_t st = (cudaStream_t)stream;
    // the gradient of the states, against time; dq's states, with time; dk's are dv's, turned
    Pass by_v = make_pass(p, rk, rq, rd, ov, true);
    Args g = common_args(p);
    g.log_decay = log_decay;
    by_v.z_in = dlast;
    if (p->split()) {
        FoldArgs f = {};
        g.n_passes = dq ? 2 : 1;
        g.pass[0] = by_v;
        local_states(p, g.pass[0], 0, !dq);
        f.first[0] = dlast, f.reverse[0] = 1;
        if (dq) {
            g.pass[1] = make_pass(p, rq, rk, rv, oq, false);
            local_states(p, g.pass[1], 1, false);
            f.first[1] = first;
        } else {
            into_summary(p, g.pass[0], dsummary);
            f.summary[0] = dsummary;
        }
        e = run(p, g, st);
        if (e == SPARBIT_OK) e = fold(p, f, g.n_passes, log_decay, st);
        if (e != SPARBIT_OK || !dq) return e;
    }
    from_segment(p, by_v, 0);
    g.pass[0] = by_v;
    into_summary(p, g.pass[0], dsummary);
    g.n_passes = 1;
    if (dq) {
        g.full = 1;
        g.n_passes = 3;
        Pass& by_k = g.pass[1] = make_pass(p, rv, rd, rq, ok, true);
        by_k.z_in = by_v.z_in, by_k.slots_in = by_v.slots_in;
        turned(by_k);
        Pass& by_q = g.pass[2] = make_pass(p, rd, rv, rk, oq, false);
        by_q.z_in = first;
        from_segment(p, by_q, 1);
        turned(by_q);
    }
    return run(p, g, st);
}

int sparbit_linear_attention_plan_status(sparbit_linear_attention_plan_t* p) {
    if (!p) return SPARBIT_ERR_ARG;
    const int e = ready(p);
    if (e != SPARBIT_OK) return e;
    CU(cudaDeviceSynchronize());
    uint32_t status;
    CU(cudaMemcpy(&status, p->work, sizeof status, cudaMemcpyDeviceToHost));
    if (status == 0) return SPARBIT_OK;
    CU(cudaMemset(p->work, 0, sizeof status));
    return SPARBIT_ERR_TIMEOUT;
}

int sparbit_linear_attention_plan_set_wait_test(sparbit_linear_attention_plan_t* p, int withhold, uint64_t timeout_ns) {
    if (!p) return SPARBIT_ERR_ARG;
    p->withhold = withhold != 0;
    p->limit = timeout_ns ? timeout_ns : kWaitNs;
    return SPARBIT_OK;
}

int sparbit_linear_attention_step(size_t rows, int heads, int key_size, int value_size, int dtype, float scale, const void* q,
                                  size_t q_ld, const void* k, size_t k_ld, const void* v, size_t v_ld, const float* log_decay,
                                  const int32_t* slots, size_t n_slots, const float* state_in, float* state_out, void* o,
                                  size_t o_ld, void* stream) {
    if (heads < 1 || key_size < 1 || value_size < 1 || !known_dtype(dtype) || !isfinite(scale)) return SPARBIT_ERR_ARG;
    if (rows == 0) return SPARBIT_OK;
    if (!q || !k || !v || !log_decay || !o || (n_slots && (!state_in || !state_out))) return SPARBIT_ERR_ARG;
    if (!slots && n_slots < rows) return SPARBIT_ERR_ARG;
    if (key_size > SPARBIT_LINEAR_ATTENTION_MAX_SIZE || value_size > SPARBIT_LINEAR_ATTENTION_MAX_SIZE || heads > 4096 ||
        rows > 0x7fffffffu / (unsigned)heads || n_slots > 0x7fffffffu)
        return SPARBIT_ERR_LIMIT;
    const size_t kw = (size_t)heads * key_size, vw = (size_t)heads * value_size, es = elem_size(dtype);
    const size_t state = kw * value_size;
    if (bad_pitch(q_ld, kw, rows) || bad_pitch(k_ld, kw, rows) || bad_pitch(v_ld, vw, rows) || bad_pitch(o_ld, vw, rows) ||
        (n_slots && state > kMostElements / n_slots))
        return SPARBIT_ERR_ARG;
    const Region rq{q, rows, kw * es, q_ld * es}, rk{k, rows, kw * es, k_ld * es}, rv{v, rows, vw * es, v_ld * es},
        rl{log_decay, 1, (size_t)heads * 4, 0}, rs{slots, 1, rows * 4, 0}, ri{state_in, 1, n_slots * state * 4, 0},
        ro{o, rows, vw * es, o_ld * es}, so{state_out, 1, n_slots * state * 4, 0};
    const Region ins[] = {rq, rk, rv, rl, rs};
    for (const Region& in : ins)
        if (regions_overlap(ro, in) || regions_overlap(so, in)) return SPARBIT_ERR_ALIAS;
    if (regions_overlap(ro, ri) || regions_overlap(ro, so) || (state_in != state_out && regions_overlap(so, ri)))
        return SPARBIT_ERR_ALIAS;
    if (misaligned(es, {q, k, v, o}) || misaligned(4, {log_decay, slots, state_in, state_out})) return SPARBIT_ERR_ARG;
    const bool wide = value_size % 4 == 0 && ((uintptr_t)state_in | (uintptr_t)state_out) % 16 == 0;
    // few rows: a head's values in slices of 32, a CTA each
    const int slice = rows * heads < 2 * (size_t)kSms && value_size > 32 ? 32 : value_size;
    const dim3 grid((unsigned)(rows * heads), (unsigned)((value_size + slice - 1) / slice));
    auto go = [&]<typename T, bool kWide>() {
        CU(launch(attention_step_kernel<T, kWide>, grid, dim3(256), 0, (cudaStream_t)stream, heads, key_size, value_size, slice,
                  scale, (const T*)q, (int64_t)q_ld, (const T*)k, (int64_t)k_ld, (const T*)v, (int64_t)v_ld, log_decay, slots,
                  (int64_t)n_slots, state_in, state_out, (T*)o, (int64_t)o_ld));
        return (int)SPARBIT_OK;
    };
    auto typed = [&]<typename T>() { return wide ? go.template operator()<T, true>() : go.template operator()<T, false>(); };
    if (dtype == SPARBIT_F32) return typed.template operator()<float>();
    if (dtype == SPARBIT_BF16) return typed.template operator()<__nv_bfloat16>();
    return typed.template operator()<__half>();
}

int sparbit_linear_attention_join(int P, int first_rank, int n_ranks, int heads, int key_size, int value_size,
                                  const float* gathered, const float* first, float* out, int reverse, void* stream) {
    if (P < 1 || first_rank < 0 || n_ranks < 1 || n_ranks > P - first_rank || heads < 1 || key_size < 1 || value_size < 1)
        return SPARBIT_ERR_ARG;
    if (!gathered || !out) return SPARBIT_ERR_ARG;
    if (key_size > SPARBIT_LINEAR_ATTENTION_MAX_SIZE || value_size > SPARBIT_LINEAR_ATTENTION_MAX_SIZE || heads > 4096 ||
        n_ranks > 65535)
        return SPARBIT_ERR_LIMIT;
    const size_t size = (size_t)key_size * value_size, block = heads * (1 + size);
    if (P * block > kMostElements / n_ranks) return SPARBIT_ERR_OVERFLOW;
    const Region rg{gathered, 1, (size_t)n_ranks * P * block * 4, 0}, rf{first, 1, heads * size * 4, 0},
        ro{out, 1, (size_t)n_ranks * heads * size * 4, 0};
    if (regions_overlap(ro, rg) || regions_overlap(ro, rf)) return SPARBIT_ERR_ALIAS;
    if (misaligned(4, {gathered, first, out})) return SPARBIT_ERR_ARG;
    CU(launch(attention_join_kernel, dim3((unsigned)((size + 255) / 256), (unsigned)heads, (unsigned)n_ranks), dim3(256), 0,
              (cudaStream_t)stream, P, first_rank, heads, (int)size, gathered, first, out, reverse));
    return SPARBIT_OK;
}

}  // extern "C"
