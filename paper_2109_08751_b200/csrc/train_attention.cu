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
#include <math.h>
#include <string.h>

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
    int32_t len, seq, id;
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
    // states: element (key, value) of head h of unit u at [u * unit + h * kd * vd + key * k_step + value * v_step]
    const float* z_in;         // null: zero
    float* z_out;              // null: not wanted
    float* decay_out;          // [u * unit_out + h]: decay over the whole sequence; null: not wanted
    int64_t unit_in, unit_out;
    int k_step, v_step;
    int in_by_segment, out_by_segment;  // units are segments, not sequences
    int skip_ends;             // what the last segment of a sequence adds is not wanted
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
// addition; a ring of two pieces of c^T, 32 tokens each in up to three parts.
constexpr uint32_t kColScore = 0, kColOut = 128, kColAdd = 256, kColC = 384, kSlotCols = 48;

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
__device__ __forceinline__ void tmem_store8(uint32_t addr, const uint32_t (&r)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(addr), "r"(r[0]),
                 "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}
__device__ __forceinline__ void tmem_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
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
    static constexpr int kParts = 3;        // parts that hold a number of 32 bits
    static constexpr uint32_t kFormat = (1u << 7) | (1u << 10), kExponent = 0x7f80u;
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
    static constexpr uint32_t kFormat = 0, kExponent = 0x7c00u;
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        const __half2 v = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
    static __device__ __forceinline__ float low(uint32_t v) { return __half2float(__ushort_as_half((unsigned short)v)); }
    static __device__ __forceinline__ float high(uint32_t v) {
        return __half2float(__ushort_as_half((unsigned short)(v >> 16)));
    }
};

// The power of two that brings `most` to 2^13 .. 2^14, as an exponent: fp16 has few, so rows of its operands are scaled.
// Numbers below 2^-27 stay below that: they make nothing that fp16 can hold.
__device__ __forceinline__ int exponent_for(float most) {
    const int e = (int)(__float_as_uint(most) >> 23 & 0xff);
    if (e == 0 || e == 255) return 0;
    const int by = 13 - (e - 127);
    return by > 40 ? 40 : by < -110 ? -110 : by;
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

constexpr int kOutWarps = 4, kStateWarps = 8, kLoadWarps = 4;
constexpr int kTensorThreads = 32 * (kOutWarps + kStateWarps + kLoadWarps + 1);

// 128 tokens of one tensor's head into panels of swizzled rows; tokens from n on and columns from `width` on are zero.
template <int kWide>
__device__ __forceinline__ void load_tile(uint32_t dst, const char* src, int64_t pitch, int width, int panels, int n, int t) {
    const int per_row = panels * 8, row0 = t / per_row, piece = t - row0 * per_row;  // 8 or 16 pieces of 16 bytes a row
    const int step = 128 / per_row;                                                   // a multiple of 8
    const uint32_t to = dst + (piece >> 3) * kPanel + row0 * 128 + (((piece & 7) ^ (row0 & 7)) << 4);
    const char* from = src + row0 * pitch + piece * 16;
    const int left = (width - piece * 8) * 2;  // bytes of this piece that the row has
#pragma unroll 8
    for (int i = 0; i < kChunk / 8; i++) {
        if (i * step >= kChunk) break;
        const int row = row0 + i * step;
        if constexpr (kWide == 16) {
            const int bytes = row < n && left > 0 ? 16 : 0;
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + i * step * 128),
                         "l"(bytes ? from + i * step * pitch : src), "r"(bytes)
                         : "memory");
        } else if constexpr (kWide >= 4) {
#pragma unroll
            for (int k = 0; k < 16; k += kWide) {
                const int bytes = row < n && left > k ? kWide : 0;
                asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(to + i * step * 128 + k),
                             "l"(bytes ? from + i * step * pitch + k : src), "n"(kWide), "r"(bytes)
                             : "memory");
            }
        } else {
            uint32_t v[4];
#pragma unroll
            for (int k = 0; k < 4; k++) {
                const unsigned short* p = reinterpret_cast<const unsigned short*>(from + i * step * pitch + k * 4);
                v[k] = row < n && left > k * 4 ? p[0] : 0u;
                if (row < n && left > k * 4 + 2) v[k] |= (uint32_t)p[1] << 16;
            }
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + i * step * 128), "r"(v[0]), "r"(v[1]),
                         "r"(v[2]), "r"(v[3])
                         : "memory");
        }
    }
}
__device__ __forceinline__ void load_any(int wide, uint32_t dst, const char* src, int64_t pitch, int width, int panels, int n,
                                         int t) {
    if (wide == 16) load_tile<16>(dst, src, pitch, width, panels, n, t);
    else if (wide == 8) load_tile<8>(dst, src, pitch, width, panels, n, t);
    else if (wide == 4) load_tile<4>(dst, src, pitch, width, panels, n, t);
    else load_tile<2>(dst, src, pitch, width, panels, n, t);
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
// First token of a chunk and the way to the next ones, in the order of the pass.
__device__ __forceinline__ int64_t first_row(const Work& k, int chunk) {
    return k.p->reverse ? k.s.row0 + k.s.len - 1 - (int64_t)chunk * kChunk : k.s.row0 + (int64_t)chunk * kChunk;
}
__device__ __forceinline__ int tokens_of(const Work& k, int chunk) {
    const int left = k.s.len - chunk * kChunk;
    return left < kChunk ? left : kChunk;
}
// Where a state goes; null where this segment leaves none.
__device__ __forceinline__ float* state_out(const Work& k) {
    const Pass& p = *k.p;
    if (!p.z_out || !(p.out_by_segment || (k.s.ends & (p.reverse ? 1 : 2)))) return nullptr;
    return p.z_out + (p.out_by_segment ? k.s.id : k.s.seq) * p.unit_out + (int64_t)k.head * p.kd * p.vd;
}
__device__ __forceinline__ const float* state_in(const Work& k) {
    const Pass& p = *k.p;
    if (!p.z_in) return nullptr;
    return p.z_in + (p.in_by_segment ? k.s.id : k.s.seq) * p.unit_in + (int64_t)k.head * p.kd * p.vd;
}
__device__ __forceinline__ void decay_out(const Work& k, const float* log_decay) {
    const Pass& p = *k.p;
    if (p.decay_out && (k.s.ends & (p.reverse ? 1 : 2)))
        p.decay_out[k.s.seq * p.unit_out + k.head] =
            k.s.seq_len ? (float)exp((double)log_decay[k.head] * (double)k.s.seq_len) : 1.0f;
}

// One CTA per SM, its warps in four roles: four write out (a token each lane), eight hold the state (a value each lane,
// half of the keys a warp), four load, one issues products.  A chunk is
//   score = a b^T;  its weights W = intra d^(i - j) score, causal, rounded to 16 bits into tensor memory
//   out = a Z (Z rounded to 16 bits in shared memory), scaled by row in tensor memory, + W c
//   add = (c times gain d^(n - e - j))^T b, the scaled c in two or three 16-bit parts that hold its 32 bits
// with Z in registers and the three chains side by side.  W and Z are the only roundings to 16 bits on the way:
// together they leave out about 1.4 times as far off as rounding it to its type does.
template <typename T>
__global__ void __launch_bounds__(kTensorThreads, 1) attention_tensor_kernel(const __grid_constant__ Args g) {
    using B = Bits<T>;
    constexpr int kParts = B::kParts, kMostStages = 4;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t bars[2 * kMostStages + 12];
    __shared__ uint32_t tmem_base, gave_up;
    __shared__ uint32_t bad[2];  // number of the last (every other) chunk whose c holds an infinity or a NaN
    __shared__ __align__(16) float left[kChunk];       // what a token's part is worth at the end of the chunk
    __shared__ short z_exp[2][kMostSize], part_exp[2][kMostSize];  // fp16: scales of Z, and of each half's share of a row
    const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t z_base = ring + g.stages * g.stage_bytes;
    const uint32_t full = smem_u32(bars), empty = full + 8 * kMostStages, scored = empty + 8 * kMostStages;
    const uint32_t weighted = scored + 8, entered = scored + 16, done = scored + 24, c_ready = scored + 32, c_free = scored + 48,
                   added = scored + 64, z_ready = scored + 72, out_free = scored + 80, met = scored + 88;
    const int warp = __shfl_sync(kAllLanes, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < g.stages; i++) bar_init(full + 8 * i, 32 * kLoadWarps), bar_init(empty + 8 * i, g.full ? kOutWarps : 1);
        bar_init(scored, 1), bar_init(weighted, kOutWarps), bar_init(entered, 1), bar_init(done, 1);
        for (int i = 0; i < 2; i++) bar_init(c_ready + 8 * i, kStateWarps), bar_init(c_free + 8 * i, 1);
        bar_init(added, 1), bar_init(z_ready, kStateWarps), bar_init(out_free, kOutWarps), bar_init(met, kStateWarps);
        gave_up = bad[0] = bad[1] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kOutWarps + kStateWarps + kLoadWarps) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base)), "r"(512)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = tmem_base;
    pdl_wait();
    pdl_trigger();
    bool ok = true;
    uint32_t c = 0;  // chunks so far, of all that this CTA works on

    if (warp < kOutWarps) {
        // ---- weights and output
        const int row = warp * 32 + lane;
        const uint32_t lanes = (uint32_t)(warp * 32) << 16;
        for (int w = blockIdx.x; w < g.total && g.full && ok; w += gridDim.x) {
            const Work k = work_of(g, w);
            const Pass& p = *k.p;
            const int panels_k = (p.kd + 63) / 64, panels_v = (p.vd + 63) / 64;
            // d^(31 - j) for the lanes of this warp; each warp has its own copy in its lanes
            const float mine = exp2f(k.l2 * (31 - lane));
            const float enter = p.inter * exp2f(k.l2 * (row + p.e));
            for (int chunk = 0; chunk < k.chunks && ok; chunk++, c++) {
                const uint32_t st = c % g.stages, stage = ring + st * g.stage_bytes;
                const int n = tokens_of(k, chunk);
                if (!warp_wait(scored, c & 1, &gave_up, g.limit)) { ok = false; break; }
                fence_after();
                int shift = 0;  // fp16: the row's weights are held times 2^shift
                if constexpr (B::kScaled) {
                    float most = 0.0f;
                    for (int b = 0; b <= warp; b++) {
                        uint32_t r[32];
                        tmem_load32(tmem + kColScore + lanes + b * 32, r);
                        const float far = p.intra * exp2f(k.l2 * (row - b * 32 - 31));
#pragma unroll
                        for (int j = 0; j < 32; j++) {
                            const float d = __shfl_sync(kAllLanes, mine, j);
                            const float weight = b < warp ? far * d : p.intra * exp2f(k.l2 * (lane >= j ? lane - j : 0));
                            if (b < warp || lane >= j) most = fmaxf(most, fabsf(__uint_as_float(r[j]) * weight));
                        }
                    }
                    shift = exponent_for(most);
                }
                const float up = power_of_two(shift);
#pragma unroll 1
                for (int b = 0; b < 4; b++) {
                    uint32_t out[16];
                    if (b < warp) {
                        uint32_t r[32];
                        tmem_load32(tmem + kColScore + lanes + b * 32, r);
                        const float far = p.intra * exp2f(k.l2 * (row - b * 32 - 31)) * up;
#pragma unroll
                        for (int j = 0; j < 16; j++) {
                            const float d0 = __shfl_sync(kAllLanes, mine, 2 * j), d1 = __shfl_sync(kAllLanes, mine, 2 * j + 1);
                            out[j] = B::pack(__uint_as_float(r[2 * j]) * (far * d0), __uint_as_float(r[2 * j + 1]) * (far * d1));
                        }
                    } else if (b == warp) {
                        uint32_t r[32];
                        tmem_load32(tmem + kColScore + lanes + b * 32, r);
#pragma unroll
                        for (int j = 0; j < 16; j++) {
                            const int i0 = lane - 2 * j, i1 = i0 - 1;
                            const float x = __uint_as_float(r[2 * j]) * (p.intra * exp2f(k.l2 * (i0 > 0 ? i0 : 0)) * up);
                            const float y = __uint_as_float(r[2 * j + 1]) * (p.intra * exp2f(k.l2 * (i1 > 0 ? i1 : 0)) * up);
                            out[j] = B::pack(i0 >= 0 ? x : 0.0f, i1 >= 0 ? y : 0.0f);
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < 16; j++) out[j] = 0u;
                    }
                    tmem_store16(tmem + kColScore + lanes + b * 16, out);
                }
                if (!warp_wait(entered, c & 1, &gave_up, g.limit)) { ok = false; break; }
                fence_after();
                const float rise = enter * up;
#pragma unroll 1
                for (int b = 0; b * 32 < p.vd; b++) {
                    uint32_t r[32];
                    tmem_load32(tmem + kColOut + lanes + b * 32, r);
#pragma unroll
                    for (int j = 0; j < 32; j++) {
                        float v = __uint_as_float(r[j]) * rise;
                        if constexpr (B::kScaled) v *= power_of_two(-z_exp[c & 1][b * 32 + j]);
                        r[j] = __float_as_uint(v);
                    }
                    tmem_store32(tmem + kColOut + lanes + b * 32, r);
                }
                tmem_store_wait();
                fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(weighted);
                if (!warp_wait(done, c & 1, &gave_up, g.limit)) { ok = false; break; }
                fence_after();
                const bool by_hand = *(volatile uint32_t*)&bad[c & 1] == c + 1;
                const float down = power_of_two(-shift);
                // out in 16 bits, over the tiles of a and b, which nobody needs any more; each warp its own rows
                const uint32_t pitch = panels_v * 128, own = stage + warp * 32 * pitch;
                const uint32_t c_tile = stage + 2 * panels_k * kPanel;
#pragma unroll 1
                for (int b = 0; b * 32 < p.vd; b++) {
                    uint32_t r[32];
                    tmem_load32(tmem + kColOut + lanes + b * 32, r);
                    if (by_hand) {
                        // c holds an infinity or a NaN, which a product would carry to the tokens in front of it (times
                        // their weight of zero): the sum over the tokens up to each row, one by one
                        for (int q = 0; q <= warp; q++) {
                            uint32_t v[16];
                            asm volatile(
                                "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
                                "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
                                "tcgen05.wait::ld.sync.aligned;"
                                : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]),
                                  "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]),
                                  "=r"(v[14]), "=r"(v[15])
                                : "r"(tmem + kColScore + lanes + q * 16)
                                : "memory");
#pragma unroll
                            for (int j = 0; j < 32; j++) {
                                const int token = q * 32 + j;
                                if (token > row) continue;
                                const float weight = j & 1 ? B::high(v[j / 2]) : B::low(v[j / 2]);
#pragma unroll 4
                                for (int x = 0; x < 32; x += 8) {
                                    const int col = b * 32 + x;
                                    uint32_t u[4];
                                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                                                 : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3])
                                                 : "r"(c_tile + (col >> 6) * kPanel + token * 128 +
                                                       ((((col >> 3) & 7) ^ (token & 7)) << 4)));
#pragma unroll
                                    for (int y = 0; y < 8; y++) {
                                        const float value = y & 1 ? B::high(u[y / 2]) : B::low(u[y / 2]);
                                        r[x + y] = __float_as_uint(fmaf(weight, value, __uint_as_float(r[x + y])));
                                    }
                                }
                            }
                        }
                    }
#pragma unroll
                    for (int j = 0; j < 32; j += 8) {
                        uint32_t v[4];
#pragma unroll
                        for (int i = 0; i < 4; i++)
                            v[i] = B::pack(__uint_as_float(r[j + 2 * i]) * down, __uint_as_float(r[j + 2 * i + 1]) * down);
                        const int piece = b * 4 + j / 8;
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(own + lane * pitch +
                                                                                      ((piece ^ (lane & 7)) << 4)),
                                     "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3])
                                     : "memory");
                    }
                }
                fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive(out_free);
                const int64_t row0 = first_row(k, chunk);
                T* const to = (T*)p.out + (int64_t)k.head * p.vd;
                if (p.out_wide == 16) {
                    const int per_row = p.vd >> 3;
                    for (int i = lane; i < 32 * per_row; i += 32) {
                        const int r = i / per_row, piece = i - r * per_row, token = warp * 32 + r;
                        if (token >= n) break;
                        uint32_t v[4];
                        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                                     : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
                                     : "r"(own + r * pitch + ((piece ^ (r & 7)) << 4))
                                     : "memory");
                        const int64_t at = p.reverse ? row0 - token : row0 + token;
                        *reinterpret_cast<uint4*>(to + at * p.out_ld + piece * 8) = make_uint4(v[0], v[1], v[2], v[3]);
                    }
                } else {
                    for (int r = 0; r < 32 && warp * 32 + r < n; r++) {
                        const int token = warp * 32 + r;
                        const int64_t at = p.reverse ? row0 - token : row0 + token;
                        for (int col = lane; col < p.vd; col += 32) {
                            unsigned short v;
                            asm volatile("ld.shared.u16 %0, [%1];"
                                         : "=h"(v)
                                         : "r"(own + r * pitch + (((col >> 3) ^ (r & 7)) << 4) + (col & 7) * 2)
                                         : "memory");
                            reinterpret_cast<unsigned short*>(to)[at * p.out_ld + col] = v;
                        }
                    }
                }
                // what was read and written here comes before the next chunk's copies
                proxy_fence();
                __syncwarp();
                if (lane == 0) bar_arrive(empty + 8 * st);
            }
        }
    } else if (warp < kOutWarps + kStateWarps) {
        // ---- the state: lane = value, half of the keys a warp
        const int quad = warp & 3, half = (warp - kOutWarps) >> 2, value = quad * 32 + lane;
        const int t = threadIdx.x - 32 * kOutWarps;
        const uint32_t lanes = (uint32_t)(quad * 32) << 16;
        uint32_t pieces = 0;  // of c^T so far
        uint32_t meetings = 0;
        // a barrier of the state's warps that gives up like every other wait
        auto meet = [&] {
            __syncwarp();
            if (lane == 0) bar_arrive(met);
            ok = ok && warp_wait(met, meetings++ & 1, &gave_up, g.limit);
        };
        for (int w = blockIdx.x; w < g.total && ok; w += gridDim.x) {
            const Work k = work_of(g, w);
            const Pass& p = *k.p;
            const int panels_k = (p.kd + 63) / 64;
            const int keys = (p.kd + 15) / 16 * 16, share = (keys / 2 + 15) / 16 * 16;
            const int key0 = half * share, mine = half ? keys - share : share;  // multiples of 16, at most 64
            const bool there = quad * 32 < p.vd, inside = value < p.vd;
            float z[64];
            const float* from = state_in(k);
#pragma unroll
            for (int i = 0; i < 64; i++) {
                const int key = key0 + i;
                z[i] = from && inside && i < mine && key < p.kd ? from[(int64_t)key * p.k_step + (int64_t)value * p.v_step] : 0.0f;
            }
            // rounds Z into shared memory for the products with a
            auto put = [&](uint32_t of) {
                float up = 1.0f;
                if constexpr (B::kScaled) {
                    float most = 0.0f;
#pragma unroll
                    for (int i = 0; i < 64; i++)
                        if (i < mine) most = fmaxf(most, fabsf(z[i]));
                    part_exp[half][value] = (short)exponent_for(most);
                    // a half of zeros (or of numbers that are none) asks for nothing
                    if (!(most > 0.0f && most < INFINITY)) part_exp[half][value] = 127;
                    meet();
                    int e = min(part_exp[0][value], part_exp[1][value]);
                    if (e == 127) e = 0;
                    if (half == 0) z_exp[of & 1][value] = (short)e;
                    up = power_of_two(e);
                    meet();
                }
                if (there) {
#pragma unroll
                    for (int i = 0; i < 64; i += 8) {
                        if (i >= mine) break;
                        const int col = key0 + i;
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(
                                         z_base + (col >> 6) * kPanel + value * 128 + ((((col >> 3) & 7) ^ (value & 7)) << 4)),
                                     "r"(B::pack(z[i] * up, z[i + 1] * up)), "r"(B::pack(z[i + 2] * up, z[i + 3] * up)),
                                     "r"(B::pack(z[i + 4] * up, z[i + 5] * up)), "r"(B::pack(z[i + 6] * up, z[i + 7] * up))
                                     : "memory");
                    }
                }
                proxy_fence();
                __syncwarp();
                if (lane == 0) bar_arrive(z_ready);
            };
            if (g.full && k.chunks) {
                // the chunk before has read its Z
                if (c > 0 && !warp_wait(entered, (c - 1) & 1, &gave_up, g.limit)) { ok = false; break; }
                put(c);
            }
            for (int chunk = 0; chunk < k.chunks && ok; chunk++, c++) {
                const uint32_t st = c % g.stages, stage = ring + st * g.stage_bytes;
                const int n = tokens_of(k, chunk);
                if (chunk == 0 || n < kChunk) {  // others are as the one before
                    meet();
                    if (t < kChunk) left[t] = t < n ? p.gain * exp2f(k.l2 * (n - p.e - t)) : 0.0f;
                    meet();
                }
                if (!warp_wait(full + 8 * st, (c / g.stages) & 1, &gave_up, g.limit)) { ok = false; break; }
                const uint32_t c_tile = stage + 2 * panels_k * kPanel;
                const uint32_t at = c_tile + (value >> 6) * kPanel + (value & 7) * 2;
                const int piece = (value >> 3) & 7;
                int shift = 0;
                if constexpr (B::kScaled) {
                    float most = 0.0f;
                    if (there) {
#pragma unroll 16
                        for (int j = 0; j < 64; j++) {
                            const int token = half * 64 + j;
                            unsigned short u;
                            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(u) : "r"(at + token * 128 + ((piece ^ (token & 7)) << 4)));
                            most = fmaxf(most, fabsf(B::low(u) * left[token]));
                        }
                    }
                    part_exp[half][value] = most > 0.0f && most < INFINITY ? (short)exponent_for(most) : (short)127;
                    meet();
                    shift = min(part_exp[0][value], part_exp[1][value]);
                    if (shift == 127) shift = 0;
                    meet();
                }
                const float up = power_of_two(shift);
                uint32_t odd = 0;
                for (int q = 0; q < 4; q++, pieces++) {
                    const uint32_t slot = pieces & 1;
                    if (pieces >= 2 && !warp_wait(c_free + 8 * slot, (pieces / 2 - 1) & 1, &gave_up, g.limit)) { ok = false; break; }
                    fence_after();
                    if (there) {
                        uint32_t part[kParts][8];
#pragma unroll
                        for (int j = 0; j < 16; j += 2) {
                            float x[2];
#pragma unroll
                            for (int i = 0; i < 2; i++) {
                                const int token = q * 32 + half * 16 + j + i;
                                unsigned short u;
                                asm volatile("ld.shared.u16 %0, [%1];"
                                             : "=h"(u)
                                             : "r"(at + token * 128 + ((piece ^ (token & 7)) << 4)));
                                odd |= (u & B::kExponent) == B::kExponent;
                                x[i] = B::low(u) * left[token] * up;
                            }
#pragma unroll
                            for (int i = 0; i < kParts; i++) {
                                part[i][j / 2] = B::pack(x[0], x[1]);
                                x[0] -= B::low(part[i][j / 2]);
                                x[1] -= B::high(part[i][j / 2]);
                            }
                        }
#pragma unroll
                        for (int i = 0; i < kParts; i++)
                            tmem_store8(tmem + kColC + slot * kSlotCols + i * 16 + half * 8 + lanes, part[i]);
                        tmem_store_wait();
                        if (q == 3 && inside && odd) *(volatile uint32_t*)&bad[c & 1] = c + 1;
                    }
                    fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive(c_ready + 8 * slot);
                }
                if (!ok || !warp_wait(added, c & 1, &gave_up, g.limit)) { ok = false; break; }
                fence_after();
                const float decay = exp2f(k.l2 * n), down = power_of_two(-shift);
                if (there) {
#pragma unroll
                    for (int b = 0; b < 4; b++) {
                        if (b * 16 >= mine) break;
                        float v[16];
                        tmem_load16(tmem + kColAdd + lanes + key0 + b * 16, v);
#pragma unroll
                        for (int i = 0; i < 16; i++) z[b * 16 + i] = fmaf(z[b * 16 + i], decay, B::kScaled ? v[i] * down : v[i]);
                    }
                    fence_before();
                }
                if (g.full && chunk + 1 < k.chunks) {
                    if (!warp_wait(entered, c & 1, &gave_up, g.limit)) { ok = false; break; }
                    put(c + 1);
                }
            }
            if (!ok) break;
            float* const to = state_out(k);
            if (to && inside) {
#pragma unroll
                for (int i = 0; i < 64; i++) {
                    const int key = key0 + i;
                    if (i < mine && key < p.kd) to[(int64_t)key * p.k_step + (int64_t)value * p.v_step] = z[i];
                }
            }
            if (t == 0) decay_out(k, g.log_decay);
        }
    } else if (warp < kOutWarps + kStateWarps + kLoadWarps) {
        // ---- loads
        const int t = threadIdx.x - 32 * (kOutWarps + kStateWarps);
        for (int w = blockIdx.x; w < g.total && ok; w += gridDim.x) {
            const Work k = work_of(g, w);
            const Pass& p = *k.p;
            const int panels_k = (p.kd + 63) / 64, panels_v = (p.vd + 63) / 64;
            const int way = p.reverse ? -2 : 2;
            for (int chunk = 0; chunk < k.chunks; chunk++, c++) {
                const uint32_t st = c % g.stages, stage = ring + st * g.stage_bytes;
                if (c >= (uint32_t)g.stages && !warp_wait(empty + 8 * st, (c / g.stages - 1) & 1, &gave_up, g.limit)) {
                    ok = false;
                    break;
                }
                const int n = tokens_of(k, chunk);
                const int64_t row = first_row(k, chunk);
                if (g.full)
                    load_any(p.a_wide, stage, (const char*)p.a + (row * p.a_ld + (int64_t)k.head * p.kd) * 2, way * p.a_ld, p.kd,
                             panels_k, n, t);
                load_any(p.b_wide, stage + panels_k * kPanel, (const char*)p.b + (row * p.b_ld + (int64_t)k.head * p.kd) * 2,
                         way * p.b_ld, p.kd, panels_k, n, t);
                load_any(p.c_wide, stage + 2 * panels_k * kPanel, (const char*)p.c + (row * p.c_ld + (int64_t)k.head * p.vd) * 2,
                         way * p.c_ld, p.vd, panels_v, n, t);
                asm volatile("cp.async.wait_all;" ::: "memory");
                proxy_fence();
                bar_arrive(full + 8 * st);
            }
        }
        // all products have reported before the CTA ends
        for (uint32_t i = c > (uint32_t)g.stages ? c - g.stages : 0; i < c && ok; i++)
            ok = warp_wait(empty + 8 * (i % g.stages), (i / g.stages) & 1, &gave_up, g.limit);
    } else {
        // ---- products
        uint32_t pieces = 0;
        bool by_hand = false;
        for (int w = blockIdx.x; w < g.total && ok; w += gridDim.x) {
            const Work k = work_of(g, w);
            const Pass& p = *k.p;
            const int panels_k = (p.kd + 63) / 64;
            const uint32_t keys = (p.kd + 15) / 16, values = (p.vd + 15) / 16;  // of 16
            constexpr uint32_t kBase = (1u << 4) | B::kFormat | (128u >> 4) << 24;
            const uint32_t score_desc = kBase | (128u >> 3) << 17, enter_desc = kBase | (values * 2) << 17,
                           out_desc = enter_desc | 1u << 16, add_desc = kBase | (keys * 2) << 17 | 1u << 16;
            for (int chunk = 0; chunk < k.chunks && ok; chunk++, c++) {
                const uint32_t st = c % g.stages, stage = ring + st * g.stage_bytes;
                const int n = tokens_of(k, chunk);
                const uint64_t a = smem_desc(stage, 16, 1024), b = smem_desc(stage + panels_k * kPanel, 16, 1024),
                               z = smem_desc(z_base, 16, 1024);
                const uint64_t b_turned = smem_desc(stage + panels_k * kPanel, kPanel, 1024),
                               c_turned = smem_desc(stage + 2 * panels_k * kPanel, kPanel, 1024);
                if (!warp_wait(full + 8 * st, (c / g.stages) & 1, &gave_up, g.limit)) { ok = false; break; }
                fence_after();
                if (g.full) {
                    // the weights of the chunk before, in the place of the scores, are used up
                    if (c > 0 && !warp_wait(done, (c - 1) & 1, &gave_up, g.limit)) { ok = false; break; }
                    if (by_hand && !warp_wait(out_free, (c - 1) & 1, &gave_up, g.limit)) { ok = false; break; }
                    fence_after();
                    if (elect_one()) {
                        for (uint32_t i = 0; i < keys; i++)
                            mma_ss(tmem + kColScore, a + (i >> 2) * (kPanel >> 4) + (i & 3) * 2, b + (i >> 2) * (kPanel >> 4) + (i & 3) * 2,
                                   score_desc, i > 0);
                        mma_done(scored);
                    }
                    __syncwarp();
                    if (c > 0 && !warp_wait(out_free, (c - 1) & 1, &gave_up, g.limit)) { ok = false; break; }
                    if (!warp_wait(z_ready, c & 1, &gave_up, g.limit)) { ok = false; break; }
                    fence_after();
                    if (elect_one()) {
                        for (uint32_t i = 0; i < keys; i++)
                            mma_ss(tmem + kColOut, a + (i >> 2) * (kPanel >> 4) + (i & 3) * 2, z + (i >> 2) * (kPanel >> 4) + (i & 3) * 2,
                                   enter_desc, i > 0);
                        mma_done(entered);
                    }
                    __syncwarp();
                }
                for (int q = 0; q < 4 && ok; q++, pieces++) {
                    const uint32_t slot = pieces & 1;
                    if (!warp_wait(c_ready + 8 * slot, (pieces / 2) & 1, &gave_up, g.limit)) { ok = false; break; }
                    fence_after();
                    if (elect_one()) {
                        // small parts first: less of them is cut off
#pragma unroll
                        for (int part = kParts - 1; part >= 0; part--)
#pragma unroll
                            for (int i = 0; i < 2; i++)
                                mma_ts(tmem + kColAdd, tmem + kColC + slot * kSlotCols + part * 16 + i * 8,
                                       b_turned + (q * 2 + i) * (2048 >> 4), add_desc, q > 0 || part < kParts - 1 || i > 0);
                        mma_done(c_free + 8 * slot);
                        if (q == 3 && !g.withhold) mma_done(added);
                        if (q == 3 && !g.full) mma_done(empty + 8 * st);
                    }
                    __syncwarp();
                }
                if (!ok) break;
                if (g.full) {
                    if (!warp_wait(weighted, c & 1, &gave_up, g.limit)) { ok = false; break; }
                    fence_after();
                    by_hand = *(volatile uint32_t*)&bad[c & 1] == c + 1;
                    if (elect_one()) {
                        if (!by_hand) {
                            const int steps = (n + 15) / 16;
                            for (int i = 0; i < steps; i++)
                                mma_ts(tmem + kColOut, tmem + kColScore + i * 8, c_turned + i * (2048 >> 4), out_desc, true);
                        }
                        mma_done(done);
                    }
                    __syncwarp();
                }
            }
        }
        for (uint32_t i = pieces > 2 ? pieces - 2 : 0; i < pieces && ok; i++)
            ok = warp_wait(c_free + 8 * (i & 1), (i / 2) & 1, &gave_up, g.limit);
        if (!ok) {  // let the products under way end before the CTA does
            const unsigned long long until = now_ns() + 1000000ull;
            while (now_ns() < until) {
            }
        }
    }
    __syncthreads();
    if (threadIdx.x == 0 && gave_up) *g.status = 2;
    if (warp == kOutWarps + kStateWarps + kLoadWarps) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
}

// ---- 32-bit types -------------------------------------------------------------------------------

// The same passes in plain 32-bit arithmetic, in chunks of 32 tokens; a CTA a segment and head, Z in shared memory.
constexpr int kPlainChunk = 32, kPlainThreads = 256;
__host__ __device__ constexpr int plain_pitch(int d) { return (d + 3) / 4 * 4 + 4; }
__host__ __device__ constexpr size_t plain_smem(int kd, int vd) {
    return sizeof(float) * ((size_t)kPlainChunk * (2 * plain_pitch(kd) + plain_pitch(vd) + kPlainChunk + 1 + 3) +
                            (size_t)(kd + 3) / 4 * 4 * plain_pitch(vd));
}
__device__ __forceinline__ void load_plain(float* dst, const float* src, int64_t pitch, int width, bool wide, int n) {
    const int p = plain_pitch(width), quads = (width + 3) / 4;
    for (int i = threadIdx.x; i < kPlainChunk * quads; i += kPlainThreads) {
        const int row = i / quads, col = (i - row * quads) * 4;
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (row < n) {
            const float* from = src + row * pitch + col;
            if (wide) {
                v = *reinterpret_cast<const float4*>(from);
            } else {
                v.x = from[0];
                if (col + 1 < width) v.y = from[1];
                if (col + 2 < width) v.z = from[2];
                if (col + 3 < width) v.w = from[3];
            }
        }
        *reinterpret_cast<float4*>(dst + row * p + col) = v;
    }
}
__device__ __forceinline__ float4 fma4(float a, float4 b, float4 c) {
    return make_float4(fmaf(a, b.x, c.x), fmaf(a, b.y, c.y), fmaf(a, b.z, c.z), fmaf(a, b.w, c.w));
}
__device__ __forceinline__ float dot4(float4 a, float4 b, float c) {
    return fmaf(a.x, b.x, fmaf(a.y, b.y, fmaf(a.z, b.z, fmaf(a.w, b.w, c))));
}
__global__ void __launch_bounds__(kPlainThreads) attention_plain_kernel(const __grid_constant__ Args g) {
    extern __shared__ __align__(16) float sm[];
    pdl_wait();
    pdl_trigger();
    const Work k = work_of(g, blockIdx.x);
    const Pass& p = *k.p;
    const int kd4 = (p.kd + 3) / 4 * 4, vd4 = (p.vd + 3) / 4 * 4, kp = plain_pitch(p.kd), vp = plain_pitch(p.vd);
    float* const a = sm;
    float* const b = a + kPlainChunk * kp;
    float* const c = b + kPlainChunk * kp;
    float* const weights = c + kPlainChunk * vp;                 // [32][36]
    float* const z = weights + kPlainChunk * (kPlainChunk + 4);  // [kd4][vp]
    const int t = threadIdx.x;
    const float* from = state_in(k);
    for (int i = t; i < kd4 * vp; i += kPlainThreads) {
        const int key = i / vp, value = i - key * vp;
        z[i] = from && key < p.kd && value < p.vd ? from[(int64_t)key * p.k_step + (int64_t)value * p.v_step] : 0.0f;
    }
    const int steps = (k.s.len + kPlainChunk - 1) / kPlainChunk;
    const int64_t way = p.reverse ? -1 : 1;
    for (int chunk = 0; chunk < steps; chunk++) {
        const int at = chunk * kPlainChunk, n = min(kPlainChunk, k.s.len - at);
        const int64_t row = p.reverse ? k.s.row0 + k.s.len - 1 - at : k.s.row0 + at;
        __syncthreads();
        if (g.full)
            load_plain(a, (const float*)p.a + row * p.a_ld + (int64_t)k.head * p.kd, way * p.a_ld, p.kd, p.a_wide == 16, n);
        load_plain(b, (const float*)p.b + row * p.b_ld + (int64_t)k.head * p.kd, way * p.b_ld, p.kd, p.b_wide == 16, n);
        load_plain(c, (const float*)p.c + row * p.c_ld + (int64_t)k.head * p.vd, way * p.c_ld, p.vd, p.c_wide == 16, n);
        __syncthreads();
        if (g.full) {
            // weights: a thread has four tokens of c for one of a
            const int i = t >> 3, j0 = t & 7;
            float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            for (int x = 0; x < kd4; x += 4) {
                const float4 u = *reinterpret_cast<const float4*>(a + i * kp + x);
#pragma unroll
                for (int y = 0; y < 4; y++) s[y] = dot4(u, *reinterpret_cast<const float4*>(b + (j0 + 8 * y) * kp + x), s[y]);
            }
#pragma unroll
            for (int y = 0; y < 4; y++) {
                const int j = j0 + 8 * y;
                weights[i * (kPlainChunk + 4) + j] = j <= i ? s[y] * (p.intra * exp2f(k.l2 * (i - j))) : 0.0f;
            }
            __syncthreads();
            // out: four tokens (every eighth) and four values a thread
            for (int v0 = (t & 31) * 4; v0 < vd4; v0 += 128) {
                const int r0 = t >> 5;
                float4 o[4];
#pragma unroll
                for (int y = 0; y < 4; y++) o[y] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                for (int x = 0; x < kd4; x += 4) {
                    float4 zz[4];
#pragma unroll
                    for (int y = 0; y < 4; y++) zz[y] = *reinterpret_cast<const float4*>(z + (x + y) * vp + v0);
#pragma unroll
                    for (int y = 0; y < 4; y++) {
                        const float4 u = *reinterpret_cast<const float4*>(a + (r0 + 8 * y) * kp + x);
                        o[y] = fma4(u.x, zz[0], fma4(u.y, zz[1], fma4(u.z, zz[2], fma4(u.w, zz[3], o[y]))));
                    }
                }
#pragma unroll
                for (int y = 0; y < 4; y++) {
                    const float f = p.inter * exp2f(k.l2 * (r0 + 8 * y + p.e));
                    o[y] = make_float4(o[y].x * f, o[y].y * f, o[y].z * f, o[y].w * f);
                }
#pragma unroll
                for (int y = 0; y < 4; y++) {
                    const int i = r0 + 8 * y;
                    // a token after this one weighs nothing, whatever it holds
                    for (int j = 0; j <= i; j++)
                        o[y] = fma4(weights[i * (kPlainChunk + 4) + j], *reinterpret_cast<const float4*>(c + j * vp + v0), o[y]);
                    if (i >= n) continue;
                    float* to = (float*)p.out + (row + way * i) * p.out_ld + (int64_t)k.head * p.vd + v0;
                    if (p.out_wide == 16) {
                        *reinterpret_cast<float4*>(to) = o[y];
                    } else {
                        to[0] = o[y].x;
                        if (v0 + 1 < p.vd) to[1] = o[y].y;
                        if (v0 + 2 < p.vd) to[2] = o[y].z;
                        if (v0 + 3 < p.vd) to[3] = o[y].w;
                    }
                }
            }
            __syncthreads();
        }
        // Z: eight keys and eight values a thread
        const float decay = exp2f(k.l2 * n);
        for (int i = t; i < kPlainChunk; i += kPlainThreads)
            weights[i] = i < n ? p.gain * exp2f(k.l2 * (n - p.e - i)) : 0.0f;
        __syncthreads();
        for (int k0 = (t >> 4) * 4; k0 < kd4; k0 += 64) {
            for (int v0 = (t & 15) * 4; v0 < vd4; v0 += 64) {
                float4 s[4];
#pragma unroll
                for (int y = 0; y < 4; y++) s[y] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                for (int j = 0; j < n; j++) {
                    const float w = weights[j];
                    float4 u = *reinterpret_cast<const float4*>(b + j * kp + k0);
                    const float4 v = *reinterpret_cast<const float4*>(c + j * vp + v0);
                    s[0] = fma4(u.x * w, v, s[0]), s[1] = fma4(u.y * w, v, s[1]);
                    s[2] = fma4(u.z * w, v, s[2]), s[3] = fma4(u.w * w, v, s[3]);
                }
#pragma unroll
                for (int y = 0; y < 4; y++) {
                    float4* to = reinterpret_cast<float4*>(z + (k0 + y) * vp + v0);
                    *to = fma4(decay, *to, s[y]);
                }
            }
        }
    }
    __syncthreads();
    float* const to = state_out(k);
    if (to)
        for (int i = t; i < p.kd * p.vd; i += kPlainThreads) {
            const int key = p.v_step == 1 ? i / p.vd : i % p.kd, value = p.v_step == 1 ? i % p.vd : i / p.kd;
            to[(int64_t)key * p.k_step + (int64_t)value * p.v_step] = z[key * vp + value];
        }
    if (t == 0) decay_out(k, g.log_decay);
}

// ---- along the segments, along the ranks, single tokens -----------------------------------------

struct FoldArgs {
    float* states[2];          // [segments][heads][size]: what each adds; on return the state that enters it
    const float* first[2];     // [sequences][heads][size], null: zero
    float* summary[2];         // null: not wanted; else the last segments' additions are there too
    int reverse[2];
    const Segment* segments;   // in the order of time
    const int32_t* begin;      // [sequences + 1]
    const float* log_decay;
    int heads, size;
};
__global__ void __launch_bounds__(256) attention_fold_kernel(const __grid_constant__ FoldArgs g) {
    pdl_wait();
    pdl_trigger();
    const int which = blockIdx.z, s = blockIdx.x / g.heads, h = blockIdx.x - s * g.heads;
    const int at = blockIdx.y * 256 + threadIdx.x;
    const int lo = g.begin[s], n = g.begin[s + 1] - lo;
    const float l2 = log2_decay(g.log_decay, h);
    const int64_t unit = (int64_t)g.heads * g.size;
    if (at < g.size) {
        float z = g.first[which] ? g.first[which][s * unit + (int64_t)h * g.size + at] : 0.0f;
        float* const states = g.states[which] + (int64_t)h * g.size + at;
        for (int i = 0; i < n; i++) {
            const int id = g.reverse[which] ? lo + n - 1 - i : lo + i;
            const bool last = i + 1 == n && !g.summary[which];
            const float here = last ? 0.0f : states[id * unit];
            states[id * unit] = z;
            z = fmaf(exp2f(l2 * (float)g.segments[id].len), z, here);
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
    bool split = false;                // some sequence has several segments
    std::vector<Segment> time, list;   // segments in the order of time, and the longest first
    std::vector<int32_t> begin;        // of each sequence's segments
    char* work = nullptr;
    int device = -1, sm_count = 0;
    unsigned long long limit = kWaitNs;
    int withhold = 0;

    size_t states() const { return (size_t)heads * kd * vd; }
    size_t block() const { return states() + heads; }
    size_t off_time() const { return 256; }
    size_t off_list() const { return off_time() + round_up(time.size() * sizeof(Segment), 256); }
    size_t off_begin() const { return off_list() + round_up(list.size() * sizeof(Segment), 256); }
    size_t off_states(int which) const {
        return off_begin() + round_up(begin.size() * sizeof(int32_t), 256) +
               (split ? which * round_up(time.size() * states() * sizeof(float), 256) : 0);
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

int run(const Plan* p, Args& g, cudaStream_t st) {
    g.total = (int)p->list.size() * p->heads * g.n_passes;
    if (p->dtype == SPARBIT_F32) {
        size_t smem = 0;
        for (int i = 0; i < g.n_passes; i++) smem = std::max(smem, plain_smem(g.pass[i].kd, g.pass[i].vd));
        CU(cudaFuncSetAttribute(attention_plain_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
        CU(launch(attention_plain_kernel, dim3(g.total), dim3(kPlainThreads), smem, st, g));
        return SPARBIT_OK;
    }
    uint32_t state = 0;
    g.stage_bytes = 0;
    for (int i = 0; i < g.n_passes; i++) {
        const uint32_t pk = (g.pass[i].kd + 63) / 64, pv = (g.pass[i].vd + 63) / 64;
        g.stage_bytes = std::max(g.stage_bytes, (2 * pk + pv) * kPanel);
        state = std::max(state, pk * kPanel);
    }
    constexpr uint32_t kRing = 14 * kPanel;  // with what the kernel declares, all that a CTA can have
    g.stages = (int)std::min<uint32_t>(4, (kRing - state) / g.stage_bytes);
    const size_t smem = kRing + 1024;
    const dim3 grid(std::min(g.total, p->sm_count));
    auto launch_it = [&](auto kernel) {
        CU(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
        CU(launch(kernel, grid, dim3(kTensorThreads), smem, st, g));
        return (int)SPARBIT_OK;
    };
    return p->dtype == SPARBIT_BF16 ? launch_it(attention_tensor_kernel<__nv_bfloat16>) : launch_it(attention_tensor_kernel<__half>);
}

int fold(const Plan* p, FoldArgs& f, int n, const float* log_decay, cudaStream_t st) {
    f.segments = (const Segment*)(p->work + p->off_time());
    f.begin = (const int32_t*)(p->work + p->off_begin());
    f.log_decay = log_decay;
    f.heads = p->heads, f.size = p->kd * p->vd;
    for (int i = 0; i < n; i++) f.states[i] = (float*)(p->work + p->off_states(i));
    CU(launch(attention_fold_kernel, dim3((unsigned)(p->n_seqs * p->heads), (unsigned)((f.size + 255) / 256), (unsigned)n),
              dim3(256), 0, st, f));
    return SPARBIT_OK;
}

// What each segment adds to a state of its direction, for fold.
void local_states(const Plan* p, Pass& x, int which, bool all) {
    x.out = nullptr;
    x.z_in = nullptr;
    x.z_out = (float*)(p->work + p->off_states(which));
    x.out_by_segment = 1;
    x.skip_ends = !all;
}
void from_segment(const Plan* p, Pass& x, int which) {
    x.z_in = (const float*)(p->work + p->off_states(which));
    x.in_by_segment = 1;
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

// Chunks of a segment, at most; chosen for the least estimated time.  Times in chunks: a launch takes the longest SM's
// chunks and about one more for each segment; the pass over states costs about half of the main one; a fold about
// four.  8 heads x 4097 tokens in segments of 3 chunks.. see the plan's table of measured sizes.
int segment_chunks(const std::vector<int64_t>& chunks, int heads) {
    int64_t longest = 0;
    for (int64_t c : chunks) longest = std::max(longest, c);
    int64_t best = longest > 0 ? longest : 1;
    double least = 1e300;
    for (int64_t len = longest; len >= 1; len = len * 3 / 4) {
        double items = 0, all = 0;
        for (int64_t c : chunks) items += (double)((c + len - 1) / len), all += (double)c;
        items *= heads, all *= heads;
        const double rounds = items <= 3 * kSms ? ceil(items / kSms) * (len + 1) : (all + items) / kSms + len * 0.5;
        const double cost = len < longest ? 1.5 * rounds + 4 : rounds;
        if (cost < least) least = cost, best = len;
    }
    return (int)best;
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
        std::vector<int64_t> chunks;
        for (int s = 0; s < n_seqs; s++) chunks.push_back((int64_t)((lengths[s] + kChunk - 1) / kChunk));
        const int len = segment_chunks(chunks, heads);
        int64_t row = 0;
        for (int s = 0; s < n_seqs; s++) {
            const int64_t n = std::max<int64_t>(1, (chunks[s] + len - 1) / len), each = (chunks[s] + n - 1) / n * kChunk;
            p->begin.push_back((int32_t)p->time.size());
            for (int64_t at = 0, first = 1; first || at < (int64_t)lengths[s]; at += each, first = 0) {
                const int64_t left = (int64_t)lengths[s] - at, here = std::min(each, left);
                p->time.push_back(Segment{row + at, (int64_t)lengths[s], (int32_t)here, s, (int32_t)p->time.size(),
                                          (at == 0 ? 1 : 0) | (here == left ? 2 : 0)});
                if (each == 0) break;
            }
            p->split = p->split || p->time.size() - p->begin.back() > 1;
            row += (int64_t)lengths[s];
        }
        p->begin.push_back((int32_t)p->time.size());
        if (p->time.size() > 0x7fffffffu / 3 / heads) {
            delete p;
            return SPARBIT_ERR_LIMIT;
        }
        p->list = p->time;
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
    char* base = (char*)dev;
    CU(cudaMemset(base, 0, 256));
    CU(cudaMemcpy(base + p->off_time(), p->time.data(), p->time.size() * sizeof(Segment), cudaMemcpyHostToDevice));
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
    if (e == SPARBIT_OK) e = ready(p);
    if (e != SPARBIT_OK || (!o && !summary)) return e;
    const cudaStream_t st = (cudaStream_t)stream;
    const Pass main = make_pass(p, rq, rk, rv, ro, false);
    Args g = common_args(p);
    g.n_passes = 1;
    g.log_decay = log_decay;
    if (p->split) {
        g.pass[0] = main;
        local_states(p, g.pass[0], 0, !o);
        e = run(p, g, st);
        FoldArgs f = {};
        f.first[0] = first;
        f.summary[0] = o ? nullptr : summary;
        if (e == SPARBIT_OK) e = fold(p, f, 1, log_decay, st);
        if (e != SPARBIT_OK || !o) return e;
    }
    g.full = o != nullptr;
    g.pass[0] = main;
    g.pass[0].z_in = first;
    if (p->split) from_segment(p, g.pass[0], 0);
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
    if (e == SPARBIT_OK) e = ready(p);
    if (e != SPARBIT_OK || (!dq && !dsummary)) return e;
    const cudaStream_t st = (cudaStream_t)stream;
    // the gradient of the states, against time; dq's states, with time; dk's are dv's, turned
    Pass by_v = make_pass(p, rk, rq, rd, ov, true);
    Args g = common_args(p);
    g.log_decay = log_decay;
    if (p->split) {
        FoldArgs f = {};
        g.n_passes = dq ? 2 : 1;
        g.pass[0] = by_v;
        local_states(p, g.pass[0], 0, !dq);
        f.first[0] = dlast, f.reverse[0] = 1;
        f.summary[0] = dq ? nullptr : dsummary;
        if (dq) {
            g.pass[1] = make_pass(p, rq, rk, rv, oq, false);
            local_states(p, g.pass[1], 1, false);
            f.first[1] = first;
        }
        e = run(p, g, st);
        if (e == SPARBIT_OK) e = fold(p, f, g.n_passes, log_decay, st);
        if (e != SPARBIT_OK || !dq) return e;
    }
    by_v.z_in = dlast;
    if (p->split) from_segment(p, by_v, 0);
    g.pass[0] = by_v;
    into_summary(p, g.pass[0], dsummary);
    g.n_passes = 1;
    if (dq) {
        g.full = 1;
        g.n_passes = 3;
        Pass& by_k = g.pass[1] = make_pass(p, rv, rd, rq, ok, true);
        by_k.z_in = by_v.z_in, by_k.in_by_segment = by_v.in_by_segment;
        turned(by_k);
        Pass& by_q = g.pass[2] = make_pass(p, rd, rv, rk, oq, false);
        by_q.z_in = first;
        if (p->split) from_segment(p, by_q, 1);
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
    const bool wide = value_size % 4 == 0 && ((uintptr_t)state_in | (uintptr_t)state_out) % 16 == 0;
    // few rows: a head's values in slices of 32, a CTA each
    const int slice = rows * heads < 4 * (size_t)kSms && value_size > 32 ? 32 : value_size;
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
    CU(launch(attention_join_kernel, dim3((unsigned)((size + 255) / 256), (unsigned)heads, (unsigned)n_ranks), dim3(256), 0,
              (cudaStream_t)stream, P, first_rank, heads, (int)size, gathered, first, out, reverse));
    return SPARBIT_OK;
}

}  // extern "C"
