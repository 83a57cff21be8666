// Root-mean-square norm of rows, with the residual's addition in front of it and 8-bit rows with scales behind it.
//
//   r = x + residual;  y = r rstd weight, rstd = 1 / sqrt(mean(r^2) + eps)
//   g = dy weight;  dx = rstd (g - u mean(g u)) + dsum, u = r rstd;  dweight = sum dy u
//
// Bytes are the floor: a row is read once, stays in registers over the reduction and is written once.  A thread has up
// to four units of eight neighbouring columns; a row belongs to 4 .. 32 lanes of a warp or to a CTA, as many threads as
// its units take, which goes from row to row with the next one's loads on their way.  32768 x 4096 bf16 with a residual
// takes 205 us forward and 185 backward, 5.2 and 5.8 TB/s: 27 instructions an element keep half of the issue slots busy.
#include <math.h>

#include <algorithm>
#include <new>

#include "train_common.cuh"

using namespace spb;

namespace {

constexpr int kUnit = 8;             // columns of a unit
constexpr int kMostThreads = 1024;   // of a row
constexpr int kShared = 256;         // threads of a CTA whose rows belong to 32 lanes or fewer
constexpr int kParts = 592;          // CTAs that sum dweight: four an SM
constexpr int kSms = 148;

struct NormArgs {
    const void *x, *residual, *weight;
    void *sum, *y;
    uint8_t* y8;
    float *scales, *rstd;
    int64_t x_ld, residual_ld, sum_ld, y_ld, y8_ld;
    int64_t rows;
    int width, lanes;                // lanes: threads of a row
    int wide, weight_wide, y8_wide;  // rows start on multiples of 16 bytes (y8: 8)
    int block, scales_ld;            // columns of a scale, 0: all
    float eps, inverse;              // inverse: 1 / width
};
struct NormBackArgs {
    const void *dy, *sum, *weight, *dsum;
    const float* rstd;
    void* dx;
    float* parts;                    // [CTAs][width], null: dweight is not wanted
    int64_t dy_ld, sum_ld, dsum_ld, dx_ld;
    int64_t rows;
    int width, lanes, wide, weight_wide;
    float inverse;  // 1 / width
};

// A unit as it lies in memory: loaded a row ahead, converted when its turn comes.
template <typename T>
struct Raw {
    static constexpr int kPacks = kUnit * sizeof(T) / 16;
    uint4 v[kPacks];
};
template <typename T>
__device__ __forceinline__ void load_raw(const T* p, int n, bool wide, Raw<T>& r) {
    if (wide && n >= kUnit) {
#pragma unroll
        for (int i = 0; i < Raw<T>::kPacks; i++) r.v[i] = reinterpret_cast<const uint4*>(p)[i];
        return;
    }
    uint32_t w[Raw<T>::kPacks * 4];
#pragma unroll
    for (int i = 0; i < Raw<T>::kPacks * 4; i++) {
        if constexpr (sizeof(T) == 4) {
            w[i] = i < n ? reinterpret_cast<const uint32_t*>(p)[i] : 0u;
        } else {
            const unsigned short* q = reinterpret_cast<const unsigned short*>(p);
            w[i] = 2 * i < n ? q[2 * i] : 0u;
            if (2 * i + 1 < n) w[i] |= (uint32_t)q[2 * i + 1] << 16;
        }
    }
#pragma unroll
    for (int i = 0; i < Raw<T>::kPacks; i++) r.v[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
}
// Pairs of numbers, for the packed 32-bit instructions: what a row costs beside its bytes is instructions.
struct Unit {
    float2 v[kUnit / 2];
};
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

__device__ __forceinline__ float2 pair_of(uint32_t v, __nv_bfloat16) {
    return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}
__device__ __forceinline__ float2 pair_of(uint32_t v, __half) { return __half22float2(reinterpret_cast<const __half2&>(v)); }
__device__ __forceinline__ uint32_t bits_of_pair(float2 v, __nv_bfloat16) {
    const __nv_bfloat162 k = __floats2bfloat162_rn(v.x, v.y);
    return reinterpret_cast<const uint32_t&>(k);
}
__device__ __forceinline__ uint32_t bits_of_pair(float2 v, __half) {
    const __half2 k = __floats2half2_rn(v.x, v.y);
    return reinterpret_cast<const uint32_t&>(k);
}
template <typename T>
__device__ __forceinline__ Unit convert(const Raw<T>& r) {
    Unit f;
#pragma unroll
    for (int i = 0; i < Raw<T>::kPacks; i++) {
        const uint32_t w[4] = {r.v[i].x, r.v[i].y, r.v[i].z, r.v[i].w};
#pragma unroll
        for (int j = 0; j < 4; j++) {
            if constexpr (sizeof(T) == 2) f.v[j] = pair_of(w[j], T());
            else (j & 1 ? f.v[i * 2 + j / 2].y : f.v[i * 2 + j / 2].x) = __uint_as_float(w[j]);
        }
    }
    return f;
}
// Rounded to the type.
template <typename T>
__device__ __forceinline__ Raw<T> round_to(const Unit& f) {
    Raw<T> r;
    if constexpr (sizeof(T) == 2) {
        r.v[0] = make_uint4(bits_of_pair(f.v[0], T()), bits_of_pair(f.v[1], T()), bits_of_pair(f.v[2], T()), bits_of_pair(f.v[3], T()));
    } else {
#pragma unroll
        for (int i = 0; i < 2; i++)
            r.v[i] = make_uint4(__float_as_uint(f.v[2 * i].x), __float_as_uint(f.v[2 * i].y), __float_as_uint(f.v[2 * i + 1].x),
                                __float_as_uint(f.v[2 * i + 1].y));
    }
    return r;
}
template <typename T>
__device__ __forceinline__ void store_raw(T* p, int n, bool wide, const Raw<T>& r) {
    if (wide && n >= kUnit) {
#pragma unroll
        for (int i = 0; i < Raw<T>::kPacks; i++) reinterpret_cast<uint4*>(p)[i] = r.v[i];
        return;
    }
#pragma unroll
    for (int i = 0; i < Raw<T>::kPacks; i++) {
        const uint32_t w[4] = {r.v[i].x, r.v[i].y, r.v[i].z, r.v[i].w};
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const int at = (i * 4 + j) * (int)(4 / sizeof(T));
            if constexpr (sizeof(T) == 4) {
                if (at < n) reinterpret_cast<uint32_t*>(p)[at] = w[j];
            } else {
                unsigned short* q = reinterpret_cast<unsigned short*>(p);
                if (at < n) q[at] = (unsigned short)w[j];
                if (at + 1 < n) q[at + 1] = (unsigned short)(w[j] >> 16);
            }
        }
    }
}

// Reductions over the threads of a row, in one order.  `sm`: a word for each warp, two sets in turn.
struct RowSum {
    static __device__ __forceinline__ float of(float a, float b) { return a + b; }
};
struct RowMax {  // of non-negative numbers; a NaN is the largest
    static __device__ __forceinline__ float of(float a, float b) {
        return __uint_as_float(max(__float_as_uint(a), __float_as_uint(b)));
    }
};
template <typename Op>
__device__ __forceinline__ float over_lanes(float v, int lanes) {
    for (int o = (lanes < 32 ? lanes : 32) / 2; o; o >>= 1) v = Op::of(v, __shfl_xor_sync(kAllLanes, v, o));
    return v;
}
template <typename Op>
__device__ __forceinline__ float over_row(float v, int lanes, float* sm, int& turn) {
    v = over_lanes<Op>(v, lanes);
    if (lanes <= 32) return v;
    const int warp = threadIdx.x >> 5, warps = lanes >> 5;
    sm += (turn ^= 32);
    if ((threadIdx.x & 31) == 0) sm[warp] = v;
    __syncthreads();
    v = sm[0];
    for (int i = 1; i < warps; i++) v = Op::of(v, sm[i]);
    return v;
}

__device__ __forceinline__ uint32_t e4m3x2(float2 v) {
    unsigned short r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(v.y), "f"(v.x));
    return r;
}

// kMost: threads of a CTA, at most; those of 256 come several to an SM.
template <typename T, typename W, int U, int kMost>
__global__ void __launch_bounds__(kMost, kMost == 256 ? (U == 4 ? 2 : 3) : 1) norm_forward_kernel(const __grid_constant__ NormArgs g) {
    __shared__ float sm[64];
    int turn = 0;
    pdl_wait();
    pdl_trigger();
    const int lanes = g.lanes, t = threadIdx.x % lanes, together = blockDim.x / lanes;
    Raw<W> weight[U];
    Raw<T> x[U], e[U];
    int left[U];  // columns from this unit's first to the end of the row
#pragma unroll
    for (int u = 0; u < U; u++) {
        left[u] = g.width - (u * lanes + t) * kUnit;
        if (g.weight && left[u] > 0) load_raw((const W*)g.weight + (u * lanes + t) * kUnit, left[u], g.weight_wide, weight[u]);
    }
    auto fetch = [&](int64_t row) {
#pragma unroll
        for (int u = 0; u < U; u++) {
            if (row >= g.rows || left[u] <= 0) continue;
            const int col = (u * lanes + t) * kUnit;
            load_raw((const T*)g.x + row * g.x_ld + col, left[u], g.wide, x[u]);
            if (g.residual) load_raw((const T*)g.residual + row * g.residual_ld + col, left[u], g.wide, e[u]);
        }
    };
    fetch((int64_t)blockIdx.x * together + threadIdx.x / lanes);
    // all threads of a CTA go round equally often
    for (int64_t row0 = (int64_t)blockIdx.x * together; row0 < g.rows; row0 += (int64_t)gridDim.x * together) {
        const int64_t row = row0 + threadIdx.x / lanes;
        const bool there = row < g.rows;
        // columns behind the row's end hold zeros throughout
        Unit r[U];
        float2 pairs = both(0.0f);
#pragma unroll
        for (int u = 0; u < U; u++) {
            if (there && left[u] > 0) {
                r[u] = convert(x[u]);
                if (g.residual) {
                    const Unit f = convert(e[u]);
#pragma unroll
                    for (int i = 0; i < kUnit / 2; i++) r[u].v[i] = add2(r[u].v[i], f.v[i]);
                    // what is kept is what is normalised
                    x[u] = round_to<T>(r[u]);
                    if constexpr (sizeof(T) == 2) r[u] = convert(x[u]);
                }
                if (g.sum) store_raw((T*)g.sum + row * g.sum_ld + (u * lanes + t) * kUnit, left[u], g.wide, x[u]);
            } else {
#pragma unroll
                for (int i = 0; i < kUnit / 2; i++) r[u].v[i] = both(0.0f);
            }
        }
        fetch(row + (int64_t)gridDim.x * together);
#pragma unroll
        for (int u = 0; u < U; u++)
#pragma unroll
            for (int i = 0; i < kUnit / 2; i++) pairs = fma2(r[u].v[i], r[u].v[i], pairs);
        const float squares = over_row<RowSum>(pairs.x + pairs.y, lanes, sm, turn);
        float rstd = rsqrtf(fmaf(squares, g.inverse, g.eps));
        const bool big = !(squares < 1e38f);
        if (lanes <= 32 ? __any_sync(kAllLanes, big) : big) {
            // squares that 32 bits do not hold: once more, scaled.  All threads that reduce together take the same way.
            float most = 0.0f;
#pragma unroll
            for (int u = 0; u < U; u++)
#pragma unroll
                for (int i = 0; i < kUnit / 2; i++) most = RowMax::of(RowMax::of(most, fabsf(r[u].v[i].x)), fabsf(r[u].v[i].y));
            most = over_row<RowMax>(most, lanes, sm, turn);
            const float by = most < INFINITY && most > 0.0f ? exp2f((float)-ilogbf(most)) : 1.0f;
            float again = 0.0f;
#pragma unroll
            for (int u = 0; u < U; u++)
#pragma unroll
                for (int i = 0; i < kUnit / 2; i++) {
                    const float2 v = mul2(r[u].v[i], both(by));
                    again = fmaf(v.x, v.x, fmaf(v.y, v.y, again));
                }
            again = over_row<RowSum>(again, lanes, sm, turn);
            if (big) rstd = by * rsqrtf(fmaf(again, g.inverse, g.eps * by * by));
        }
        if (g.rstd && there && t == 0) g.rstd[row] = rstd;
#pragma unroll
        for (int u = 0; u < U; u++) {
            if (!there || left[u] <= 0) continue;
#pragma unroll
            for (int i = 0; i < kUnit / 2; i++) r[u].v[i] = mul2(r[u].v[i], both(rstd));
            if (g.weight) {
                const Unit w = convert(weight[u]);
#pragma unroll
                for (int i = 0; i < kUnit / 2; i++) r[u].v[i] = mul2(r[u].v[i], w.v[i]);
            }
            if (g.y) store_raw((T*)g.y + row * g.y_ld + (u * lanes + t) * kUnit, left[u], g.wide, round_to<T>(r[u]));
        }
        if (!g.y8) continue;
        float unit_most[U], row_most = 0.0f;
#pragma unroll
        for (int u = 0; u < U; u++) {
            unit_most[u] = 0.0f;
#pragma unroll
            for (int i = 0; i < kUnit / 2; i++)
                unit_most[u] = RowMax::of(RowMax::of(unit_most[u], fabsf(r[u].v[i].x)), fabsf(r[u].v[i].y));
            row_most = RowMax::of(row_most, unit_most[u]);
        }
        if (!g.block) row_most = over_row<RowMax>(row_most, lanes, sm, turn);
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int col = (u * lanes + t) * kUnit;
            float most = g.block ? over_lanes<RowMax>(unit_most[u], min(g.block / kUnit, lanes)) : row_most;
            if (!there || left[u] <= 0) continue;
            if (most < 1e-30f) most = 1e-30f;
            const float scale = most / 448.0f;
            if (g.block ? col % g.block == 0 : col == 0) g.scales[row * g.scales_ld + (g.block ? col / g.block : 0)] = scale;
            // y / scale as a reader of both forms it: y times the inverse, and what that leaves of y once more (a step of
            // Newton's method; 143 us for 16384 x 5000 f16, 134 without it).  Negated, so that a zero keeps its sign through
            // the step; no step over an infinite scale.
            const float by = -__fdividef(1.0f, scale), back = scale < INFINITY ? scale : 0.0f;
            uint32_t pairs8[kUnit / 2];
#pragma unroll
            for (int i = 0; i < kUnit / 2; i++) {
                const float2 q = mul2(r[u].v[i], both(by));
                pairs8[i] = e4m3x2(fma2(fma2(q, both(back), r[u].v[i]), both(by), q));
            }
            const uint2 q = make_uint2((pairs8[0] | pairs8[1] << 16) ^ 0x80808080u, (pairs8[2] | pairs8[3] << 16) ^ 0x80808080u);
            uint8_t* to = g.y8 + row * g.y8_ld + col;
            if (g.y8_wide && left[u] >= kUnit) {
                *reinterpret_cast<uint2*>(to) = q;
            } else {
#pragma unroll
                for (int i = 0; i < kUnit; i++)
                    if (i < left[u]) to[i] = (uint8_t)((i < 4 ? q.x : q.y) >> (i & 3) * 8);
            }
        }
    }
}

template <typename T, typename W, int U, int kMost>
__global__ void __launch_bounds__(kMost, kMost == 256 ? 2 : 1) norm_backward_kernel(const __grid_constant__ NormBackArgs g) {
    extern __shared__ float partial[];
    __shared__ float sm[64];
    int turn = 0;
    pdl_wait();
    pdl_trigger();
    const int lanes = g.lanes, t = threadIdx.x % lanes, together = blockDim.x / lanes;
    Raw<W> weight[U];
    Raw<T> raw_d[U], raw_x[U], raw_m[U];
    float next_rstd = 0.0f;
    Unit dw[U];
    int left[U];
#pragma unroll
    for (int u = 0; u < U; u++) {
        left[u] = g.width - (u * lanes + t) * kUnit;
        if (g.weight && left[u] > 0) load_raw((const W*)g.weight + (u * lanes + t) * kUnit, left[u], g.weight_wide, weight[u]);
#pragma unroll
        for (int i = 0; i < kUnit / 2; i++) dw[u].v[i] = both(0.0f);
    }
    auto fetch = [&](int64_t row) {
        next_rstd = row < g.rows ? g.rstd[row] : 0.0f;
#pragma unroll
        for (int u = 0; u < U; u++) {
            if (row >= g.rows || left[u] <= 0) continue;
            const int col = (u * lanes + t) * kUnit;
            load_raw((const T*)g.dy + row * g.dy_ld + col, left[u], g.wide, raw_d[u]);
            load_raw((const T*)g.sum + row * g.sum_ld + col, left[u], g.wide, raw_x[u]);
            if (g.dsum) load_raw((const T*)g.dsum + row * g.dsum_ld + col, left[u], g.wide, raw_m[u]);
        }
    };
    fetch((int64_t)blockIdx.x * together + threadIdx.x / lanes);
    for (int64_t row0 = (int64_t)blockIdx.x * together; row0 < g.rows; row0 += (int64_t)gridDim.x * together) {
        const int64_t row = row0 + threadIdx.x / lanes;
        const bool there = row < g.rows;
        const float rstd = next_rstd;
        Unit d[U], x[U];
        Raw<T> more[U];
#pragma unroll
        for (int u = 0; u < U; u++) {
            if (!there || left[u] <= 0) continue;
            d[u] = convert(raw_d[u]);
            x[u] = convert(raw_x[u]);
            more[u] = raw_m[u];
        }
        fetch(row + (int64_t)gridDim.x * together);
        float2 inner = both(0.0f);
#pragma unroll
        for (int u = 0; u < U; u++) {
            if (!there || left[u] <= 0) continue;
#pragma unroll
            for (int i = 0; i < kUnit / 2; i++) {
                x[u].v[i] = mul2(x[u].v[i], both(rstd));
                dw[u].v[i] = fma2(d[u].v[i], x[u].v[i], dw[u].v[i]);
            }
            if (g.weight) {
                const Unit w = convert(weight[u]);
#pragma unroll
                for (int i = 0; i < kUnit / 2; i++) d[u].v[i] = mul2(d[u].v[i], w.v[i]);
            }
#pragma unroll
            for (int i = 0; i < kUnit / 2; i++) inner = fma2(d[u].v[i], x[u].v[i], inner);
        }
        const float mean = over_row<RowSum>(inner.x + inner.y, lanes, sm, turn) * g.inverse;
#pragma unroll
        for (int u = 0; u < U; u++) {
            if (!there || left[u] <= 0) continue;
            Unit m;
            if (g.dsum) {
                m = convert(more[u]);
            } else {
#pragma unroll
                for (int i = 0; i < kUnit / 2; i++) m.v[i] = both(0.0f);
            }
#pragma unroll
            for (int i = 0; i < kUnit / 2; i++)
                d[u].v[i] = fma2(both(rstd), fma2(x[u].v[i], both(-mean), d[u].v[i]), m.v[i]);
            store_raw((T*)g.dx + row * g.dx_ld + (u * lanes + t) * kUnit, left[u], g.wide, round_to<T>(d[u]));
        }
    }
    if (!g.parts) return;
    float* const out = g.parts + (int64_t)blockIdx.x * g.width;
    if (together == 1) {
#pragma unroll
        for (int u = 0; u < U; u++)
            if (left[u] > 0) store_raw(out + (u * lanes + t) * kUnit, left[u], g.width % 4 == 0, round_to<float>(dw[u]));
        return;
    }
    const int columns = U * lanes * kUnit;
#pragma unroll
    for (int u = 0; u < U; u++)
#pragma unroll
        for (int i = 0; i < kUnit; i++)
            partial[(threadIdx.x / lanes) * columns + (u * lanes + t) * kUnit + i] = i & 1 ? dw[u].v[i / 2].y : dw[u].v[i / 2].x;
    __syncthreads();
    for (int col = threadIdx.x; col < g.width; col += blockDim.x) {
        float s = 0.0f;
        for (int i = 0; i < together; i++) s += partial[i * columns + col];
        out[col] = s;
    }
}

// dweight from the CTAs' sums, always added in the same order.
__global__ void __launch_bounds__(256) norm_weight_kernel(const float* __restrict__ parts, int n, int width,
                                                          float* __restrict__ dweight) {
    __shared__ float sm[8][33];
    pdl_wait();
    pdl_trigger();
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5, col = blockIdx.x * 32 + x;
    float s = 0.0f;
    if (col < width)
#pragma unroll 8
        for (int i = y; i < n; i += 8) s += parts[(int64_t)i * width + col];
    sm[y][x] = s;
    __syncthreads();
    if (y == 0 && col < width) {
        for (int i = 1; i < 8; i++) s += sm[i][x];
        dweight[col] = s;
    }
}

}  // namespace

struct sparbit_norm_plan_s {
    int width = 0, dtype = 0, weight_dtype = 0, block = 0;
    float eps = 0.0f;
    char* work = nullptr;
    int device = -1;
    size_t work_bytes() const { return (size_t)kParts * width * sizeof(float); }
};

namespace {

using Plan = sparbit_norm_plan_s;

// Threads of a row, units of a thread, the most threads that the kernel is built for, CTAs an SM holds.  With few rows a
// thread has one unit, which is done soonest.  With many, two or four and the next row's on their way keep enough loads in
// flight; the registers that they take (80, or 128 from four units and backward) leave room for so many CTAs.  Four units do
// not fit everywhere: backward above 8192 columns (16384) spills 0.8 to 1.9 KB a thread (2.0 to 2.9), forward above 16384 0.9 to
// 1.5 KB, which costs two to seven times the bytes' time: 8192 x 12288 bf16 335 us backward and 145 forward, of 125;
// 4096 x 20000 726 and 311, of 101; 2048 x 32768 689 and 250, of 83 (8192 x 8192: 105 and 90, of 83).
struct Shape {
    int lanes, units, threads, most, per_sm;
};
Shape shape_of(const Plan* p, size_t rows, bool backward) {
    const int all = (p->width + kUnit - 1) / kUnit;
    Shape s;
    if (all <= 32) {
        s.lanes = 4, s.units = 1;
        while (s.lanes < all) s.lanes *= 2;
    } else {
        if (all <= kMostThreads && rows < 4 * kSms) s.units = 1;
        else s.units = all <= (backward ? 1024 : 512) ? 2 : 4;
        s.lanes = ((all + s.units - 1) / s.units + 31) / 32 * 32;
    }
    s.threads = s.lanes <= 32 ? kShared : s.lanes;
    s.most = s.threads <= 256 ? 256 : s.units > 1 && s.threads <= 512 ? 512 : kMostThreads;
    s.per_sm = std::max(1, (s.most > 256 ? s.most : backward || s.units == 4 ? 512 : 768) / s.threads);
    return s;
}

// f.operator()<T, W, U, kMost>() for the plan's types and a shape, those that shape_of gives.
template <bool kBackward, typename T, typename W, typename Fn>
int by_shape(const Shape& s, Fn f) {
    if (s.units == 1)
        return s.most == 256 ? f.template operator()<T, W, 1, 256>() : f.template operator()<T, W, 1, 1024>();
    if (s.units == 2) {
        if constexpr (kBackward)
            if (s.most == 512) return f.template operator()<T, W, 2, 512>();
        return f.template operator()<T, W, 2, 256>();
    }
    if constexpr (!kBackward)
        if (s.most == 256) return f.template operator()<T, W, 4, 256>();
    return s.most == 512 ? f.template operator()<T, W, 4, 512>() : f.template operator()<T, W, 4, 1024>();
}
template <bool kBackward, typename Fn>
int by_types(const Plan* p, const Shape& s, Fn f) {
    if (p->dtype == SPARBIT_F32) return by_shape<kBackward, float, float>(s, f);
    if (p->dtype == SPARBIT_BF16)
        return p->weight_dtype == SPARBIT_F32 ? by_shape<kBackward, __nv_bfloat16, float>(s, f)
                                              : by_shape<kBackward, __nv_bfloat16, __nv_bfloat16>(s, f);
    return p->weight_dtype == SPARBIT_F32 ? by_shape<kBackward, __half, float>(s, f) : by_shape<kBackward, __half, __half>(s, f);
}

Region region(const Plan* p, const void* x, size_t rows, size_t ld) {
    const size_t es = elem_size(p->dtype);
    return Region{x, rows, p->width * es, ld * es};
}

}  // namespace

extern "C" {

int sparbit_norm_plan_create(size_t width, int dtype, int weight_dtype, float eps, int block, sparbit_norm_plan_t** out) {
    if (!out) return SPARBIT_ERR_ARG;
    *out = nullptr;
    if (width < 1 || !known_dtype(dtype) || (weight_dtype != SPARBIT_F32 && weight_dtype != dtype) || !(eps >= 1e-30f) ||
        !isfinite(eps))
        return SPARBIT_ERR_ARG;
    if (block != 0 && block != 32 && block != 64 && block != 128 && block != 256) return SPARBIT_ERR_ARG;
    if (width > SPARBIT_NORM_MAX_WIDTH) return SPARBIT_ERR_LIMIT;
    Plan* p = new (std::nothrow) Plan();
    if (!p) return SPARBIT_ERR_NOMEM;
    p->width = (int)width, p->dtype = dtype, p->weight_dtype = weight_dtype, p->eps = eps, p->block = block;
    *out = p;
    return SPARBIT_OK;
}

int sparbit_norm_plan_destroy(sparbit_norm_plan_t* p) {
    delete p;
    return SPARBIT_OK;
}

size_t sparbit_norm_plan_workspace_bytes(const sparbit_norm_plan_t* p) { return p ? p->work_bytes() : 0; }

int sparbit_norm_plan_set_workspace(sparbit_norm_plan_t* p, void* dev, size_t bytes) {
    if (!p) return SPARBIT_ERR_ARG;
    if (!dev || bytes < p->work_bytes() || (uintptr_t)dev % 16) return SPARBIT_ERR_WORKSPACE;
    p->work = nullptr;
    CU(cudaGetDevice(&p->device));
    p->work = (char*)dev;
    return SPARBIT_OK;
}

int sparbit_norm_forward(sparbit_norm_plan_t* p, size_t rows, const void* x, size_t x_ld, const void* residual,
                         size_t residual_ld, const void* weight, void* sum, size_t sum_ld, void* y, size_t y_ld, void* y8,
                         size_t y8_ld, float* scales, float* rstd, void* stream) {
    if (!p || !y8 != !scales) return SPARBIT_ERR_ARG;
    if (rows == 0) return SPARBIT_OK;
    const size_t w = p->width, es = elem_size(p->dtype), ws = elem_size(p->weight_dtype);
    if (!x) return SPARBIT_ERR_ARG;
    if (rows > 0x7fffffffu) return SPARBIT_ERR_LIMIT;
    if (bad_pitch(x_ld, w, rows) || (residual && bad_pitch(residual_ld, w, rows)) || (sum && bad_pitch(sum_ld, w, rows)) ||
        (y && bad_pitch(y_ld, w, rows)) || (y8 && bad_pitch(y8_ld, w, rows)))
        return SPARBIT_ERR_ARG;
    const size_t per_row = p->block ? (w + p->block - 1) / p->block : 1;
    const Region rx = region(p, x, rows, x_ld), rr = region(p, residual, rows, residual_ld), rw{weight, 1, w * ws, 0},
                 rs = region(p, sum, rows, sum_ld), ry = region(p, y, rows, y_ld), r8{y8, rows, w, y8_ld},
                 rc{scales, 1, rows * per_row * 4, 0}, rt{rstd, 1, rows * 4, 0};
    const Region outs[] = {rs, ry, r8, rc, rt};
    for (int i = 0; i < 5; i++) {
        if (regions_overlap(outs[i], rw)) return SPARBIT_ERR_ALIAS;
        if (!(i == 0 && sum == x && sum_ld == x_ld) && regions_overlap(outs[i], rx)) return SPARBIT_ERR_ALIAS;
        if (!(i == 0 && sum == residual && sum_ld == residual_ld) && regions_overlap(outs[i], rr)) return SPARBIT_ERR_ALIAS;
        for (int j = 0; j < i; j++)
            if (regions_overlap(outs[i], outs[j])) return SPARBIT_ERR_ALIAS;
    }
    if (misaligned(es, {x, residual, sum, y}) || misaligned(ws, {weight}) || misaligned(4, {scales, rstd})) return SPARBIT_ERR_ARG;
    if (!sum && !y && !y8 && !rstd) return SPARBIT_OK;
    NormArgs g = {};
    g.x = x, g.residual = residual, g.weight = weight, g.sum = sum, g.y = y, g.y8 = (uint8_t*)y8;
    g.scales = scales, g.rstd = rstd;
    g.x_ld = (int64_t)x_ld, g.residual_ld = (int64_t)residual_ld, g.sum_ld = (int64_t)sum_ld, g.y_ld = (int64_t)y_ld;
    g.y8_ld = (int64_t)y8_ld;
    g.rows = (int64_t)rows, g.width = (int)w;
    const uintptr_t bits = (uintptr_t)x | x_ld * es | (residual ? (uintptr_t)residual | residual_ld * es : 0) |
                           (sum ? (uintptr_t)sum | sum_ld * es : 0) | (y ? (uintptr_t)y | y_ld * es : 0);
    g.wide = bits % 16 == 0;
    g.weight_wide = (uintptr_t)weight % 16 == 0;
    g.y8_wide = ((uintptr_t)y8 | y8_ld) % 8 == 0;
    g.block = p->block, g.scales_ld = (int)per_row, g.eps = p->eps, g.inverse = 1.0f / (float)w;
    const Shape s = shape_of(p, rows, false);
    g.lanes = s.lanes;
    const size_t together = s.threads / s.lanes, grid = std::min((size_t)(kSms * s.per_sm), (rows + together - 1) / together);
    return by_types<false>(p, s, [&]<typename T, typename W, int U, int kMost>() {
        CU(launch(norm_forward_kernel<T, W, U, kMost>, dim3((unsigned)grid), dim3(s.threads), 0, (cudaStream_t)stream, g));
        return (int)SPARBIT_OK;
    });
}

int sparbit_norm_backward(sparbit_norm_plan_t* p, size_t rows, const void* dy, size_t dy_ld, const void* sum,
                          size_t sum_ld, const void* weight, const float* rstd, const void* dsum, size_t dsum_ld, void* dx,
                          size_t dx_ld, float* dweight, void* stream) {
    if (!p) return SPARBIT_ERR_ARG;
    const size_t w = p->width, es = elem_size(p->dtype), ws = elem_size(p->weight_dtype);
    if (rows && (!dy || !sum || !rstd || !dx)) return SPARBIT_ERR_ARG;
    if (rows > 0x7fffffffu) return SPARBIT_ERR_LIMIT;
    if (bad_pitch(dy_ld, w, rows) || bad_pitch(sum_ld, w, rows) || bad_pitch(dx_ld, w, rows) ||
        (dsum && bad_pitch(dsum_ld, w, rows)))
        return SPARBIT_ERR_ARG;
    const Region ry = region(p, dy, rows, dy_ld), rs = region(p, sum, rows, sum_ld), rw{weight, 1, w * ws, 0},
                 rt{rstd, 1, rows * 4, 0}, rd = region(p, dsum, rows, dsum_ld), rx = region(p, dx, rows, dx_ld),
                 rg{dweight, 1, w * 4, 0}, rk{p->work, 1, p->work_bytes(), 0};
    for (const Region& in : {rs, rw, rt, rk})
        if (regions_overlap(rx, in) || regions_overlap(rg, in)) return SPARBIT_ERR_ALIAS;
    if ((!(dx == dy && dx_ld == dy_ld) && regions_overlap(rx, ry)) || (!(dx == dsum && dx_ld == dsum_ld) && regions_overlap(rx, rd)) ||
        regions_overlap(rg, ry) || regions_overlap(rg, rd) || regions_overlap(rg, rx))
        return SPARBIT_ERR_ALIAS;
    if (misaligned(es, {dy, sum, dsum, dx}) || misaligned(ws, {weight}) || misaligned(4, {rstd, dweight})) return SPARBIT_ERR_ARG;
    if (dweight) {
        if (!p->work) return SPARBIT_ERR_WORKSPACE;
        int cur = -1;
        CU(cudaGetDevice(&cur));
        if (cur != p->device) return SPARBIT_ERR_ARG;
    }
    NormBackArgs g = {};
    g.dy = dy, g.sum = sum, g.weight = weight, g.dsum = dsum, g.rstd = rstd, g.dx = dx;
    g.parts = dweight ? (float*)p->work : nullptr;
    g.dy_ld = (int64_t)dy_ld, g.sum_ld = (int64_t)sum_ld, g.dsum_ld = (int64_t)dsum_ld, g.dx_ld = (int64_t)dx_ld;
    g.rows = (int64_t)rows, g.width = (int)w, g.inverse = 1.0f / (float)w;
    const uintptr_t bits = (uintptr_t)dy | dy_ld * es | (uintptr_t)sum | sum_ld * es | (uintptr_t)dx | dx_ld * es |
                           (dsum ? (uintptr_t)dsum | dsum_ld * es : 0);
    g.wide = bits % 16 == 0;
    g.weight_wide = (uintptr_t)weight % 16 == 0;
    const Shape s = shape_of(p, rows, true);
    g.lanes = s.lanes;
    const size_t together = s.threads / s.lanes;
    const int grid = (int)std::min<size_t>(std::min(kParts, kSms * s.per_sm), (rows + together - 1) / together);
    if (grid > 0) {
        const size_t smem = together > 1 ? sizeof(float) * s.threads * s.units * kUnit : 0;
        const int e = by_types<true>(p, s, [&]<typename T, typename W, int U, int kMost>() {
            CU(launch(norm_backward_kernel<T, W, U, kMost>, dim3(grid), dim3(s.threads), smem, (cudaStream_t)stream, g));
            return (int)SPARBIT_OK;
        });
        if (e != SPARBIT_OK) return e;
    }
    if (dweight)
        CU(launch(norm_weight_kernel, dim3((unsigned)((w + 31) / 32)), dim3(256), 0, (cudaStream_t)stream,
                  (const float*)p->work, grid, (int)w, dweight));
    return SPARBIT_OK;
}

}  // extern "C"
