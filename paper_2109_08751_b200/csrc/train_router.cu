// Router: softmax over the experts' logits, the k largest, per-expert counts, balance loss and the
// gradient of the logits.
//
// L lanes of a warp share a token (8, 16 or 32, whichever holds the experts with 16 bytes of logits a
// lane, at least k), each with C runs of V = 16 bytes / element neighbouring experts.  The choice: every
// lane sorts its keys once (networks, lists of up to 8), then k times the largest head of the group
// wins and its list moves up.  A key holds the logit's order and, below it, the complement of the
// expert's index, so that keys differ and equal logits go to the lowest index.  Instructions bound
// this: 440 a token forward and 245 backward at 256 bf16 experts, k = 8 (56738 tokens: 37 us and 20 us at
// 66 % and 64 % of the issue slots, where the 29 MB of logits would take 4.5 us to read).
#include <float.h>
#include <math.h>

#include <new>
#include <type_traits>
#include <vector>

#include "train_common.cuh"

using namespace spb;

namespace {

constexpr int kWarps = 8;
constexpr int kMaxExperts = SPARBIT_ROUTER_MAX_EXPERTS;
constexpr int kMaxK = SPARBIT_ROUTER_MAX_K;
// CTAs a forward or backward pass is cut into (and one more a rank, at most): what four CTAs on each
// of a B200's 148 SMs hold at once, so that there is no second round of a few
constexpr int kSlices = 584;
constexpr float kLog2e = 1.4426950408889634f;
// Forward, p = exp2((l - top) log2(e)): what the largest logit is does not matter.  Backward it is exp2(l log2(e) -
// lse log2(e)), in which the rounding of lse and of its product stay: an error of p of 2^-16 at |lse| = kFarLse.
// Tokens beyond find top and sum again, out of the common path (56738 x 256 bf16 backward 20.0 us with the vote for
// that, 19.3 without; forward 37.3 us subtracting first, 36.9 as exp2(l log2(e) - top log2(e))).
constexpr float kFarLse = 128.0f;

// Up to so many choices are drawn by unrolled code, in which a lane's list gets shorter with every draw.
constexpr int kUnrolled = 8;
// A run of tokens of one rank, worked on by one CTA.
struct Slice {
    int32_t row0, rows, rank, pad;
};

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ float rcp_fast(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Keys: 32 bits (order of a 16-bit logit, complement of the index) or 64.  Zeros of either sign are
// equal.  A key below kLeast (-inf, or what a NaN is made into) cannot be chosen.
template <typename T>
using Key = std::conditional_t<sizeof(T) == 2, uint32_t, unsigned long long>;
template <typename T>
constexpr Key<T> kLeast = std::is_same_v<T, float>           ? (Key<T>)0x00800000ull << (sizeof(T) == 2 ? 0 : 32)
                          : std::is_same_v<T, __nv_bfloat16> ? (Key<T>)0x00800000u
                                                             : (Key<T>)0x04000000u;
__device__ __forceinline__ uint32_t plus_zero(__nv_bfloat16 a, __nv_bfloat16 b) {
    const __nv_bfloat162 r = __hadd2(__halves2bfloat162(a, b), __float2bfloat162_rn(0.0f));
    return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t plus_zero(__half a, __half b) {
    const __half2 r = __hadd2(__halves2half2(a, b), __float2half2_rn(0.0f));
    return *reinterpret_cast<const uint32_t*>(&r);
}
template <typename T>
__device__ __forceinline__ int key_index(Key<T> k) {
    if constexpr (sizeof(T) == 2) return (int)(0xffffu - (k & 0xffffu));
    else return (int)(0xffffffffu - (uint32_t)k);
}
template <typename T>
__device__ __forceinline__ float key_value(Key<T> k) {
    if constexpr (sizeof(T) == 2) {
        const uint32_t o = k >> 16;
        const unsigned short b = (unsigned short)((o & 0x8000u) ? o & 0x7fffu : ~o);
        if constexpr (std::is_same_v<T, __half>) return __half2float(__ushort_as_half(b));
        else return __bfloat162float(__ushort_as_bfloat16(b));
    } else {
        const uint32_t o = (uint32_t)(k >> 32);
        return __uint_as_float((o & 0x80000000u) ? o & 0x7fffffffu : ~o);
    }
}

template <typename K>
__device__ __forceinline__ void order(K& a, K& b) {
    const K hi = max(a, b), lo = min(a, b);
    a = hi;
    b = lo;
}
// Largest first.
template <typename K>
__device__ __forceinline__ void sort_keys(K (&k)[4]) {
    order(k[0], k[1]), order(k[2], k[3]), order(k[0], k[2]), order(k[1], k[3]), order(k[1], k[2]);
}
template <typename K>
__device__ __forceinline__ void sort_keys(K (&k)[8]) {  // odd-even merges
    order(k[0], k[1]), order(k[2], k[3]), order(k[4], k[5]), order(k[6], k[7]);
    order(k[0], k[2]), order(k[1], k[3]), order(k[4], k[6]), order(k[5], k[7]);
    order(k[1], k[2]), order(k[5], k[6]);
    order(k[0], k[4]), order(k[1], k[5]), order(k[2], k[6]), order(k[3], k[7]);
    order(k[2], k[4]), order(k[3], k[5]);
    order(k[1], k[2]), order(k[3], k[4]), order(k[5], k[6]);
}

// Over the L lanes that share a token.
template <int L>
__device__ __forceinline__ uint32_t group_max(uint32_t k) {
    if constexpr (L == 32) return __reduce_max_sync(kAllLanes, k);
#pragma unroll
    for (int o = L / 2; o; o >>= 1) k = max(k, __shfl_xor_sync(kAllLanes, k, o));
    return k;
}
template <int L>
__device__ __forceinline__ unsigned long long group_max(unsigned long long k) {
    const uint32_t hi = group_max<L>((uint32_t)(k >> 32));
    const uint32_t lo = group_max<L>((uint32_t)(k >> 32) == hi ? (uint32_t)k : 0u);
    return (unsigned long long)hi << 32 | lo;
}
template <int L>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
    for (int o = L / 2; o; o >>= 1) v += __shfl_xor_sync(kAllLanes, v, o);
    return v;
}

// A lane's logits of a row; -inf where there is no expert.  kWide, where rows start on multiples of 16
// bytes: experts (c L + l) V + i, 16 bytes a load.  Otherwise every L-th expert from l on, so that the
// lanes' single elements lie next to one another.
template <typename T, int L, int C, bool kWide>
struct Row {
    static constexpr int V = 16 / sizeof(T), N = V * C;
    Pack<T, V> run[C];
    __device__ __forceinline__ static int expert(int l, int n) { return kWide ? (n / V * L + l) * V + n % V : n * L + l; }
    __device__ __forceinline__ void load(const T* p, int l, int E, bool on) {
        const T none = from_float<T>(-INFINITY);
#pragma unroll
        for (int c = 0; c < C; c++) {
            if (kWide && on && expert(l, c * V) + V <= E) {
                run[c] = *reinterpret_cast<const Pack<T, V>*>(p + expert(l, c * V));
            } else {
#pragma unroll
                for (int i = 0; i < V; i++) run[c].v[i] = none;
                if (on) {
#pragma unroll
                    for (int i = 0; i < V; i++)
                        if (expert(l, c * V + i) < E) run[c].v[i] = p[expert(l, c * V + i)];
                }
            }
        }
    }
    __device__ __forceinline__ static void store(T* p, int l, int E, const float (&d)[N]) {
#pragma unroll
        for (int c = 0; c < C; c++) {
            if (kWide && expert(l, c * V) + V <= E) {
                Pack<T, V> o;
#pragma unroll
                for (int i = 0; i < V; i++) o.v[i] = from_float<T>(d[c * V + i]);
                *reinterpret_cast<Pack<T, V>*>(p + expert(l, c * V)) = o;
            } else {
#pragma unroll
                for (int i = 0; i < V; i++)
                    if (expert(l, c * V + i) < E) p[expert(l, c * V + i)] = from_float<T>(d[c * V + i]);
            }
        }
    }
    // A token that is left out: whatever was loaded, no expert can be chosen.  (Loading does not wait for
    // the mask.)
    __device__ __forceinline__ void leave_out() {
        const T none = from_float<T>(-INFINITY);
#pragma unroll
        for (int n = 0; n < N; n++) run[n / V].v[n % V] = none;
    }
    __device__ __forceinline__ float value(int n) const { return to_float(run[n / V].v[n % V]); }
    // Keys of all logits; a NaN with a clear sign bit comes out above everything.
    __device__ __forceinline__ void keys(int l, Key<T> (&key)[N]) const {
#pragma unroll
        for (int c = 0; c < C; c++) {
            if constexpr (sizeof(T) == 2) {
#pragma unroll
                for (int i = 0; i < V; i += 2) {
                    // two at a time: adding zero makes -0 a 0, then the sign decides which bits turn
                    const uint32_t u = plus_zero(run[c].v[i], run[c].v[i + 1]);
                    const uint32_t o = u ^ (((u >> 15) & 0x00010001u) * 0x7fffu | 0x80008000u);
                    key[c * V + i] = o << 16 | (0xffffu - (uint32_t)expert(l, c * V + i));
                    key[c * V + i + 1] = (o & 0xffff0000u) | (0xffffu - (uint32_t)expert(l, c * V + i + 1));
                }
            } else {
#pragma unroll
                for (int i = 0; i < V; i++) {
                    const uint32_t u = __float_as_uint(run[c].v[i] + 0.0f);
                    const uint32_t o = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
                    key[c * V + i] = (unsigned long long)o << 32 | (0xffffffffu - (uint32_t)expert(l, c * V + i));
                }
            }
        }
    }
};

// Two CTAs per SM with up to 16 experts a lane: 32768 x 257 bf16, k = 8, 44 us, with one 62; 32768 x 257 f32,
// k = 12, 81 us, with one 110.  One with 32: 8192 x 1000 bf16 32 us, with two 36.
template <typename T, int L, int C, bool kWide>
__global__ void __launch_bounds__(kWarps * 32, C == 1 ? 4 : C * 16 / sizeof(T) <= 16 ? 2 : 1) router_forward_kernel(const Slice* slices, const T* logits, int64_t ld,
                                                                    const uint8_t* mask, int E, int k,
                                                                    int renormalize, int32_t* indices, float* weights,
                                                                    float* lse_out, int32_t* part_counts,
                                                                    float* part_sums) {
    using R = Row<T, L, C, kWide>;
    using K = Key<T>;
    constexpr int N = R::N, kGroups = 32 / L;  // tokens of a warp
    constexpr int kList = N < 8 ? N : 8;       // keys of a sorted list
    constexpr int kSpan = N * L;               // experts there is room for
    __shared__ int32_t s_count[kSpan + 1];
    __shared__ float s_sum[kWarps * kGroups][kSpan + 1];
    pdl_wait();
    pdl_trigger();
    const Slice sl = slices[blockIdx.x];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, l = lane % L, group = w * kGroups + lane / L;
    for (int e = threadIdx.x; e <= kSpan; e += kWarps * 32) s_count[e] = 0;
    __syncthreads();
    float acc[N], z = 0.0f;
    int taken = 0;
#pragma unroll
    for (int i = 0; i < N; i++) acc[i] = 0.0f;
    R now;
    int on_byte = group < sl.rows;  // the mask's byte, looked at when the token's turn comes
    now.load(logits + ((int64_t)sl.row0 + group) * ld, l, E, on_byte);
    if (mask && on_byte) on_byte = mask[(int64_t)sl.row0 + group];
    for (int t = group; t - lane / L < sl.rows; t += kWarps * kGroups) {
        const int64_t row = (int64_t)sl.row0 + t;
        const bool inside = t < sl.rows;
        // the next token's logits travel while this one's are worked on
        const int t2 = t + kWarps * kGroups;
        int next_byte = t2 < sl.rows;
        R next;
        next.load(logits + ((int64_t)sl.row0 + t2) * ld, l, E, next_byte);
        if (mask && next_byte) next_byte = mask[(int64_t)sl.row0 + t2];
        const bool on = on_byte != 0;
        if (!on) now.leave_out();
        K key[N], head, first;
        now.keys(l, key);
        auto largest_head = [&]() {
            K most = key[0];
#pragma unroll
            for (int q = kList; q < N; q += kList) most = max(most, key[q]);
            return most;
        };
        auto find_first = [&]() {
#pragma unroll
            for (int q = 0; q < N; q += kList) sort_keys(reinterpret_cast<K(&)[kList]>(key[q]));
            head = largest_head();
            first = group_max<L>(head);
        };
        find_first();
        float p[N], sum, top;  // top: 0 where no expert can be chosen
        auto softmax = [&]() {
            const float largest = first >= kLeast<T> ? key_value<T>(first) : -INFINITY;
            top = largest > -INFINITY ? largest : 0.0f;  // +inf stays: inf - inf is the NaN it should be
            sum = 0.0f;
#pragma unroll
            for (int i = 0; i < N; i++) {
                p[i] = exp2_fast((now.value(i) - top) * kLog2e);
                sum += p[i];
            }
            sum = group_sum<L>(sum);
        };
        softmax();
        bool nan = sum != sum;
        if (__any_sync(kAllLanes, nan)) {  // a NaN somewhere in the warp's tokens: not to be chosen
            now.keys(l, key);
#pragma unroll
            for (int i = 0; i < N; i++)
                if (now.value(i) != now.value(i)) key[i] = 0;
            find_first();
            softmax();
            nan = sum != sum;
        }
        const bool part = on && (first >= kLeast<T> || nan);
        const float inv = rcp_fast(sum);
        // the chosen ones: lane j gets the j-th
        K mine = 0, won = first;
        auto draw = [&](int j, int left) {  // left: draws that may follow
            if (l == j) mine = won;
#pragma unroll
            for (int q = 0; q < N; q += kList) {
                if (key[q] == won) {
#pragma unroll
                    for (int i = 0; i < kList; i++)
                        if (i < left) key[q + i] = i + 1 < kList ? key[q + i + 1] : 0;
                }
            }
            head = largest_head();
            if (j + 1 < k) won = group_max<L>(head);
        };
        if (k <= kUnrolled) {
#pragma unroll
            for (int j = 0; j < kUnrolled; j++) {
                if (j >= k) break;
                draw(j, kUnrolled - 1 - j);
            }
        } else {
            for (int j = 0; j < k; j++) draw(j, kList);
        }
        const int index = part && mine >= kLeast<T> ? key_index<T>(mine) : -1;
        float wgt = 0.0f;
        if (index >= 0) {
            wgt = exp2_fast((key_value<T>(mine) - top) * kLog2e) * inv;
            atomicAdd(&s_count[index], 1);
        }
        if (renormalize) {
            const float chosen = group_sum<L>(wgt);
            // The quotient, and what it leaves divided once more (a Newton step): one choice has a weight of exactly 1
            // then, and no gradient.  The division itself would cost 8 % (56738 x 256 bf16 40.4 us).
            if (index >= 0) {
                const float r = rcp_fast(chosen), q = wgt * r;
                wgt = fmaf(fmaf(-q, chosen, wgt), r, q);
            }
        }
        const float lse = part ? fmaf(__log2f(sum), 0.6931471805599453f, top) : 0.0f;
        if (part) {
#pragma unroll
            for (int i = 0; i < N; i++) acc[i] = fmaf(p[i], inv, acc[i]);
            z = fmaf(lse, lse, z);
            taken++;
        }
        if (inside) {
            if (l < k) {
                indices[row * k + l] = index;
                weights[row * k + l] = wgt;
            }
            if (l == 0) lse_out[row] = lse;
        }
        now = next;
        on_byte = next_byte;
    }
    if (l == 0 && taken) atomicAdd(&s_count[kSpan], taken);
#pragma unroll
    for (int i = 0; i < N; i++) s_sum[group][R::expert(l, i)] = acc[i];
    if (l == 0) s_sum[group][kSpan] = z;
    __syncthreads();
    for (int e = threadIdx.x; e <= E; e += kWarps * 32) {
        const int at = e < E ? e : kSpan;
        float v = 0.0f;
#pragma unroll 8
        for (int u = 0; u < kWarps * kGroups; u++) v += s_sum[u][at];
        part_counts[(int64_t)blockIdx.x * (E + 1) + e] = s_count[at];
        part_sums[(int64_t)blockIdx.x * (E + 1) + e] = v;
    }
}

// Partial results of each rank's slices, added in a fixed order: 32 warps take every 32nd slice of 32
// experts, then each adds one expert's.  (Every 8th slice by 8 warps: one rank's 32768 x 256 bf16 forward
// 26 us against 31.)
constexpr int kReducers = 32;
__global__ void __launch_bounds__(32 * kReducers) router_reduce_kernel(const int2* ranks, int E, const int32_t* part_counts,
                                                                       const float* part_sums, int32_t* counts,
                                                                       float* sums) {
    __shared__ int32_t s_c[kReducers][33];
    __shared__ float s_v[kReducers][33];
    pdl_wait();
    pdl_trigger();
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5, e = blockIdx.x * 32 + x;
    const int2 r = ranks[blockIdx.y];  // first slice, number of slices
    int32_t c = 0;
    float v = 0.0f;
    if (e <= E) {
#pragma unroll 8
        for (int i = y; i < r.y; i += kReducers) {
            c += part_counts[(int64_t)(r.x + i) * (E + 1) + e];
            v += part_sums[(int64_t)(r.x + i) * (E + 1) + e];
        }
    }
    s_c[y][x] = c;
    s_v[y][x] = v;
    __syncthreads();
    c = __reduce_add_sync(kAllLanes, s_c[x][y]);
    v = group_sum<32>(s_v[x][y]);
    const int mine = blockIdx.x * 32 + y;
    if (x == 0 && mine <= E) {
        counts[(int64_t)blockIdx.y * (E + 1) + mine] = c;
        sums[(int64_t)blockIdx.y * (E + 1) + mine] = v;
    }
}

// Sum over the gathered blocks of one expert's count, or (e = E) of the tokens that take part.
__device__ __forceinline__ int64_t gathered_count(const int32_t* gathered, int G, int E, int e) {
    int64_t c = 0;
#pragma unroll 8
    for (int g = 0; g < G; g++) c += gathered[(int64_t)g * (E + 1) + e];
    return c;
}

__global__ void __launch_bounds__(256) router_balance_kernel(const int32_t* gathered, int G, int E, int k,
                                                            const float* sums, float alpha, float beta, float* loss) {
    __shared__ float s[8];
    pdl_wait();
    pdl_trigger();
    gathered += (int64_t)blockIdx.x * G * (E + 1);
    sums += (int64_t)blockIdx.x * (E + 1);
    const int64_t n = gathered_count(gathered, G, E, E);
    const float number = (float)(n > 0 ? n : 1);
    float v = 0.0f;
    for (int e = threadIdx.x; e < E; e += 256)
        v += (float)gathered_count(gathered, G, E, e) / (number * k) * sums[e];
    v = group_sum<32>(v);
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 8; i++) v += s[i];
        // squares that 32 bits do not hold count only where they have a weight
        loss[blockIdx.x] = alpha * E / number * v + (beta != 0.0f ? beta / number * sums[E] : 0.0f);
    }
}

template <typename T, int L, int C, bool kWide>
__global__ void __launch_bounds__(kWarps * 32, C == 1 ? 4 : 1) router_backward_kernel(const Slice* slices, const T* logits, int64_t ld,
                                                                     const uint8_t* mask, int E, int k,
                                                                     int renormalize, const int32_t* indices,
                                                                     const float* weights, const float* lse_in,
                                                                     const int32_t* gathered, int G,
                                                                     const float* dweights, float alpha, float beta,
                                                                     const float* dloss, T* dlogits, int64_t dld) {
    using R = Row<T, L, C, kWide>;
    constexpr int N = R::N, kGroups = 32 / L, kSpan = N * L;
    __shared__ __align__(16) float s_extra[kWarps * kGroups][kSpan];  // what the chosen weights add to a token's gradient
    __shared__ float s_f[kSpan];
    __shared__ float s_number;
    pdl_wait();
    pdl_trigger();
    const Slice sl = slices[blockIdx.x];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, l = lane % L, group = w * kGroups + lane / L;
    gathered += (int64_t)sl.rank * G * (E + 1);
    if (threadIdx.x == 0) {
        const int64_t n = gathered_count(gathered, G, E, E);
        s_number = (float)(n > 0 ? n : 1);
    }
    for (int e = threadIdx.x; e < kSpan; e += kWarps * 32)
        s_f[e] = e < E ? (float)gathered_count(gathered, G, E, e) : 0.0f;
    for (int i = threadIdx.x; i < kWarps * kGroups * kSpan; i += kWarps * 32) (&s_extra[0][0])[i] = 0.0f;
    __syncthreads();
    const float number = s_number, scale = dloss ? *dloss : 1.0f;
    const float ca = scale * alpha * E / number, cb = scale * 2.0f * beta / number;
    float f[N];
#pragma unroll
    for (int i = 0; i < N; i++) f[i] = s_f[R::expert(l, i)] / (number * k);

    struct Token {
        R row;
        int on;  // the mask's byte, looked at when the token's turn comes
        float lse, wgt, dw;
        int at;
    };
    auto fetch = [&](int t, Token& x) {
        const int64_t row = (int64_t)sl.row0 + t;
        const bool inside = t < sl.rows;
        x.row.load(logits + row * ld, l, E, inside);
        x.on = inside;
        if (mask && inside) x.on = mask[row];
        x.lse = inside ? lse_in[row] : 0.0f;
        x.at = -1;
        x.wgt = x.dw = 0.0f;
        if (inside && l < k) {
            x.at = indices[row * k + l];
            x.wgt = weights[row * k + l];
            if (dweights) x.dw = dweights[row * k + l];
        }
    };
    Token now, next;
    fetch(group, now);
    for (int t = group; t - lane / L < sl.rows; t += kWarps * kGroups) {
        fetch(t + kWarps * kGroups, next);
        if (!now.on) now.row.leave_out();
        if (now.at < 0 || now.at >= E) now.at = -1, now.dw = 0.0f;
        // a token that is left out has p = 0 and nothing chosen: its gradient comes out as 0
        float p[N], inner = 0.0f;
        const float from = now.lse * kLog2e;
#pragma unroll
        for (int i = 0; i < N; i++) {
            p[i] = exp2_fast(fmaf(now.row.value(i), kLog2e, -from));
            inner = fmaf(p[i], f[i], inner);
        }
        if (__any_sync(kAllLanes, fabsf(now.lse) > kFarLse)) {
            float top = -INFINITY, sum = 0.0f, e[N];
#pragma unroll
            for (int i = 0; i < N; i++) top = fmaxf(top, now.row.value(i));
#pragma unroll
            for (int o = L / 2; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(kAllLanes, top, o));
#pragma unroll
            for (int i = 0; i < N; i++) {
                e[i] = exp2_fast((now.row.value(i) - top) * kLog2e);
                sum += e[i];
            }
            sum = group_sum<L>(sum);
            if (fabsf(now.lse) > kFarLse) {
                const float inv = rcp_fast(sum);
                inner = 0.0f;
#pragma unroll
                for (int i = 0; i < N; i++) {
                    p[i] = e[i] * inv;
                    inner = fmaf(p[i], f[i], inner);
                }
            }
        }
        inner = group_sum<L>(inner);
        const float dwsum = group_sum<L>(now.dw * now.wgt);
        if (now.at >= 0) s_extra[group][now.at] = now.wgt * (renormalize ? now.dw - dwsum : now.dw);
        __syncwarp();
        const float common = cb * now.lse - ca * inner - (renormalize ? 0.0f : dwsum);
        if (t < sl.rows) {
            float d[N];
#pragma unroll
            for (int i = 0; i < N; i++)
                d[i] = fmaf(p[i], fmaf(ca, f[i], common), s_extra[group][R::expert(l, i)]);
            R::store(dlogits + ((int64_t)sl.row0 + t) * dld, l, E, d);
        }
        __syncwarp();
        if (now.at >= 0) s_extra[group][now.at] = 0.0f;
        __syncwarp();
        now = next;
    }
}

}  // namespace

struct sparbit_router_plan_s {
    int n_ranks = 0, E = 0, k = 0, dtype = 0, renormalize = 0;
    size_t rows = 0;
    std::vector<Slice> slices;
    std::vector<int2> ranks;
    char* work = nullptr;
    int device = -1;

    size_t off_ranks() const { return round_up(slices.size() * sizeof(Slice), 256); }
    size_t off_counts() const { return off_ranks() + round_up(ranks.size() * sizeof(int2), 256); }
    size_t off_sums() const { return off_counts() + round_up(slices.size() * (E + 1) * 4, 256); }
    size_t work_bytes() const { return off_sums() + round_up(slices.size() * (E + 1) * 4, 256); }
};

namespace {

int ready(const sparbit_router_plan_s* p) {
    if (!p->work) return SPARBIT_ERR_WORKSPACE;
    int cur = -1;
    CU(cudaGetDevice(&cur));
    return cur == p->device ? SPARBIT_OK : SPARBIT_ERR_ARG;
}

// Lanes a token and runs of 16 bytes a lane: the fewest lanes that hold the experts in one run and
// have one for each choice, then more runs.
template <typename T, bool kWide, typename F>
int by_experts(int E, int k, F f) {
    constexpr int V = 16 / sizeof(T);
    if (E <= 8 * V && k <= 8) return f.template operator()<T, 8, 1, kWide>();
    if (E <= 16 * V && k <= 16) return f.template operator()<T, 16, 1, kWide>();
    if (E <= 32 * V) return f.template operator()<T, 32, 1, kWide>();
    if (E <= 64 * V) return f.template operator()<T, 32, 2, kWide>();
    if (E <= 128 * V) return f.template operator()<T, 32, 4, kWide>();
    if constexpr (V == 4) return f.template operator()<T, 32, 8, kWide>();
    return SPARBIT_ERR_LIMIT;
}
template <typename F>
int by_type(int dtype, int E, int k, bool wide, F f) {
    switch (dtype) {
        case SPARBIT_F32: return wide ? by_experts<float, true>(E, k, f) : by_experts<float, false>(E, k, f);
        case SPARBIT_BF16:
            return wide ? by_experts<__nv_bfloat16, true>(E, k, f) : by_experts<__nv_bfloat16, false>(E, k, f);
        default: return wide ? by_experts<__half, true>(E, k, f) : by_experts<__half, false>(E, k, f);
    }
}
bool wide_rows(const void* p, size_t ld, size_t es) { return common_alignment((uintptr_t)p | ld * es, 16) == 16; }

}  // namespace

extern "C" {

int sparbit_router_plan_create(int n_ranks, const size_t* tokens, int experts, int k, int dtype, int renormalize,
                               sparbit_router_plan_t** out) {
    if (!out) return SPARBIT_ERR_ARG;
    *out = nullptr;
    if (!tokens || n_ranks < 1 || experts < 1 || k < 1 || k > experts || !known_dtype(dtype)) return SPARBIT_ERR_ARG;
    if (experts > kMaxExperts || k > kMaxK || n_ranks > 65535) return SPARBIT_ERR_LIMIT;
    size_t rows = 0;
    for (int r = 0; r < n_ranks; r++) {
        if (tokens[r] > 0x7fffffffu - rows) return SPARBIT_ERR_LIMIT;
        rows += tokens[r];
    }
    sparbit_router_plan_s* p = new (std::nothrow) sparbit_router_plan_s();
    if (!p) return SPARBIT_ERR_NOMEM;
    try {
        p->n_ranks = n_ranks;
        p->E = experts;
        p->k = k;
        p->dtype = dtype;
        p->renormalize = renormalize != 0;
        p->rows = rows;
        size_t each = (rows + kSlices - 1) / kSlices;
        each = round_up(each > 32 ? each : 32, kWarps);
        size_t row = 0;
        for (int r = 0; r < n_ranks; r++) {
            const int first = (int)p->slices.size();
            for (size_t t = 0; t < tokens[r]; t += each) {
                const size_t left = tokens[r] - t;
                p->slices.push_back(Slice{(int32_t)(row + t), (int32_t)(left < each ? left : each), r, 0});
            }
            p->ranks.push_back(make_int2(first, (int)p->slices.size() - first));
            row += tokens[r];
        }
    } catch (const std::bad_alloc&) {
        delete p;
        return SPARBIT_ERR_NOMEM;
    }
    *out = p;
    return SPARBIT_OK;
}

int sparbit_router_plan_destroy(sparbit_router_plan_t* p) {
    delete p;
    return SPARBIT_OK;
}

size_t sparbit_router_plan_workspace_bytes(const sparbit_router_plan_t* p) { return p ? p->work_bytes() : 0; }

int sparbit_router_plan_set_workspace(sparbit_router_plan_t* p, void* dev, size_t bytes) {
    if (!p) return SPARBIT_ERR_ARG;
    if (!dev || bytes < p->work_bytes() || (uintptr_t)dev % 16) return SPARBIT_ERR_WORKSPACE;
    p->work = nullptr;
    CU(cudaGetDevice(&p->device));
    if (!p->slices.empty())
        CU(cudaMemcpy(dev, p->slices.data(), p->slices.size() * sizeof(Slice), cudaMemcpyHostToDevice));
    CU(cudaMemcpy((char*)dev + p->off_ranks(), p->ranks.data(), p->ranks.size() * sizeof(int2), cudaMemcpyHostToDevice));
    CU(cudaDeviceSynchronize());
    p->work = (char*)dev;
    return SPARBIT_OK;
}

int sparbit_router_forward(sparbit_router_plan_t* p, const void* logits, size_t ld, const uint8_t* mask,
                           int32_t* indices, float* weights, float* lse, int32_t* counts, float* sums, void* stream) {
    if (!p || !counts || !sums || bad_pitch(ld, p->E, p->rows)) return SPARBIT_ERR_ARG;
    if (p->rows && (!logits || !indices || !weights || !lse)) return SPARBIT_ERR_ARG;
    const size_t es = elem_size(p->dtype), block = (size_t)p->n_ranks * (p->E + 1) * 4;
    const Region ins[] = {{logits, p->rows, p->E * es, ld * es}, {mask, 1, p->rows, 0}, {p->work, 1, p->work_bytes(), 0}};
    const Region outs[] = {{indices, 1, p->rows * p->k * 4, 0}, {weights, 1, p->rows * p->k * 4, 0},
                           {lse, 1, p->rows * 4, 0}, {counts, 1, block, 0}, {sums, 1, block, 0}};
    for (int i = 0; i < 5; i++) {
        for (const Region& in : ins)
            if (regions_overlap(outs[i], in)) return SPARBIT_ERR_ALIAS;
        for (int j = 0; j < i; j++)
            if (regions_overlap(outs[i], outs[j])) return SPARBIT_ERR_ALIAS;
    }
    const int e = ready(p);
    if (e != SPARBIT_OK) return e;
    const cudaStream_t st = (cudaStream_t)stream;
    int32_t* pc = (int32_t*)(p->work + p->off_counts());
    float* ps = (float*)(p->work + p->off_sums());
    if (!p->slices.empty()) {
        const int rc = by_type(p->dtype, p->E, p->k, wide_rows(logits, ld, es), [&]<typename T, int L, int C, bool kWide>() {
            CU(launch(router_forward_kernel<T, L, C, kWide>, dim3((unsigned)p->slices.size()), dim3(kWarps * 32), 0, st,
                      (const Slice*)p->work, (const T*)logits, (int64_t)ld, mask, p->E, p->k,
                      p->renormalize, indices, weights, lse, pc, ps));
            return (int)SPARBIT_OK;
        });
        if (rc != SPARBIT_OK) return rc;
    }
    CU(launch(router_reduce_kernel, dim3((unsigned)(p->E / 32 + 1), (unsigned)p->n_ranks), dim3(32 * kReducers), 0, st,
              (const int2*)(p->work + p->off_ranks()), p->E, (const int32_t*)pc, (const float*)ps, counts, sums));
    return SPARBIT_OK;
}

int sparbit_router_balance(sparbit_router_plan_t* p, const int32_t* gathered, int G, const float* sums, float alpha,
                           float beta, float* loss, void* stream) {
    if (!p || !gathered || !sums || !loss || G < 1) return SPARBIT_ERR_ARG;
    const size_t block = (size_t)p->n_ranks * (p->E + 1) * 4;
    const Region rl{loss, 1, (size_t)p->n_ranks * 4, 0}, rg{gathered, 1, block * G, 0}, rs{sums, 1, block, 0};
    if (regions_overlap(rl, rg) || regions_overlap(rl, rs)) return SPARBIT_ERR_ALIAS;
    CU(launch(router_balance_kernel, dim3((unsigned)p->n_ranks), dim3(256), 0, (cudaStream_t)stream, gathered, G, p->E,
              p->k, sums, alpha, beta, loss));
    return SPARBIT_OK;
}

int sparbit_router_backward(sparbit_router_plan_t* p, const void* logits, size_t ld, const uint8_t* mask,
                            const int32_t* indices, const float* weights, const float* lse, const int32_t* gathered,
                            int G, const float* dweights, float alpha, float beta, const float* dloss, void* dlogits,
                            size_t dlogits_ld, void* stream) {
    if (!p || !gathered || G < 1 || bad_pitch(ld, p->E, p->rows) || bad_pitch(dlogits_ld, p->E, p->rows))
        return SPARBIT_ERR_ARG;
    if (p->rows && (!logits || !indices || !weights || !lse || !dlogits)) return SPARBIT_ERR_ARG;
    const size_t es = elem_size(p->dtype);
    const Region out{dlogits, p->rows, p->E * es, dlogits_ld * es};
    const Region ins[] = {{logits, p->rows, p->E * es, ld * es}, {mask, 1, p->rows, 0},
                          {indices, 1, p->rows * p->k * 4, 0}, {weights, 1, p->rows * p->k * 4, 0},
                          {lse, 1, p->rows * 4, 0},
                          {gathered, 1, (size_t)p->n_ranks * G * (p->E + 1) * 4, 0},
                          {dweights, 1, p->rows * p->k * 4, 0}, {dloss, 1, 4, 0}, {p->work, 1, p->work_bytes(), 0}};
    for (const Region& in : ins)
        if (regions_overlap(out, in)) return SPARBIT_ERR_ALIAS;
    const int e = ready(p);
    if (e != SPARBIT_OK) return e;
    if (p->slices.empty()) return SPARBIT_OK;
    const bool wide = wide_rows(logits, ld, es) && wide_rows(dlogits, dlogits_ld, es);
    return by_type(p->dtype, p->E, p->k, wide, [&]<typename T, int L, int C, bool kWide>() {
        CU(launch(router_backward_kernel<T, L, C, kWide>, dim3((unsigned)p->slices.size()), dim3(kWarps * 32), 0,
                  (cudaStream_t)stream, (const Slice*)p->work, (const T*)logits, (int64_t)ld,
                  mask, p->E, p->k, p->renormalize, indices, weights, lse, gathered, G, dweights, alpha, beta, dloss,
                  (T*)dlogits, (int64_t)dlogits_ld));
        return (int)SPARBIT_OK;
    });
}

}  // extern "C"
