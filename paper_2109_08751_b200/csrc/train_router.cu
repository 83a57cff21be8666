// Router: softmax over the experts' logits, the k largest, per-expert counts, balance loss and the
// gradient of the logits.  One warp per token; a lane holds every 32nd expert's logit.
#include <float.h>
#include <math.h>

#include <new>
#include <vector>

#include "train_common.cuh"

using namespace spb;

namespace {

constexpr int kWarps = 8;
constexpr int kMaxExperts = SPARBIT_ROUTER_MAX_EXPERTS;
constexpr int kMaxK = SPARBIT_ROUTER_MAX_K;
// CTAs a forward or backward pass is cut into, at most
constexpr int kSlices = 592;

// A run of tokens of one rank, worked on by one CTA.
struct Slice {
    int32_t row0, rows, rank, pad;
};

// Order of floats as unsigned integers; NaN and -inf become 0, the key of "cannot be chosen".
__device__ __forceinline__ unsigned order_key(float v) {
    if (!(v > -INFINITY)) return 0u;
    const unsigned b = __float_as_uint(v + 0.0f);  // -0 counts as 0
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float key_value(unsigned k) {
    return __uint_as_float((k & 0x80000000u) ? (k & 0x7fffffffu) : ~k);
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(kAllLanes, v, o);
    return v;
}

// S: logits a lane holds (experts <= 32 S).  Leaves partial[slice][E+1] of counts and of sums.
template <typename T, int S>
__global__ void __launch_bounds__(kWarps * 32) router_forward_kernel(const Slice* slices, const T* logits, int64_t ld,
                                                                    const uint8_t* mask, int E, int k, int renormalize,
                                                                    int32_t* indices, float* weights, float* lse_out,
                                                                    int32_t* part_counts, float* part_sums) {
    __shared__ int32_t s_count[kMaxExperts + 1];
    __shared__ float s_sum[kWarps][32 * S + 1];
    pdl_wait();
    const Slice sl = slices[blockIdx.x];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    for (int e = threadIdx.x; e <= E; e += kWarps * 32) s_count[e] = 0;
    __syncthreads();
    float acc[S], z = 0.0f;
    int taken = 0;
#pragma unroll
    for (int i = 0; i < S; i++) acc[i] = 0.0f;
    for (int t = w; t < sl.rows; t += kWarps) {
        const int64_t row = (int64_t)sl.row0 + t;
        bool on = !mask || mask[row] != 0;
        float l[S];
        unsigned key[S];
        bool nan = false;
#pragma unroll
        for (int i = 0; i < S; i++) {
            const int e = i * 32 + lane;
            l[i] = on && e < E ? to_float(logits[row * ld + e]) : -INFINITY;
            key[i] = order_key(l[i]);
            nan |= l[i] != l[i];
        }
        nan = __any_sync(kAllLanes, nan);
        int my_index = -1;
        float my_logit = -INFINITY, top = -INFINITY;
        for (int j = 0; j < k; j++) {
            unsigned best = 0;
#pragma unroll
            for (int i = 0; i < S; i++) best = max(best, key[i]);
            best = __reduce_max_sync(kAllLanes, best);
            if (best == 0) break;  // nothing left to choose
            unsigned at = 0xffffffffu;
#pragma unroll
            for (int i = S - 1; i >= 0; i--)
                if (key[i] == best) at = i * 32 + lane;
            at = __reduce_min_sync(kAllLanes, at);
#pragma unroll
            for (int i = 0; i < S; i++)
                if (i * 32 + lane == at) key[i] = 0;
            if (j == 0) top = key_value(best);
            if (lane == j) my_index = (int)at, my_logit = key_value(best);
        }
        on = on && (top > -INFINITY || nan);
        float sum = 0.0f, p[S], lse = 0.0f;
        if (on) {
            const float from = top < INFINITY ? top : 0.0f;  // +inf: inf - inf below is the NaN it should be
#pragma unroll
            for (int i = 0; i < S; i++) {
                p[i] = i * 32 + lane < E ? expf(l[i] - from) : 0.0f;
                sum += p[i];
            }
            sum = warp_sum(sum);
            lse = from + logf(sum);
            const float inv = 1.0f / sum;
#pragma unroll
            for (int i = 0; i < S; i++) acc[i] += p[i] * inv;
            if (lane == 0) z += lse * lse, taken++;
        }
        float wgt = on && my_index >= 0 ? expf(my_logit - lse) : 0.0f;
        if (renormalize) {
            const float all = warp_sum(wgt);
            wgt = my_index >= 0 ? wgt / all : 0.0f;
        }
        if (nan && on && my_index >= 0) wgt = NAN;
        if (on && my_index >= 0) atomicAdd(&s_count[my_index], 1);
        if (lane < k) {
            indices[row * k + lane] = on ? my_index : -1;
            weights[row * k + lane] = wgt;
        }
        if (lane == 0) lse_out[row] = lse;
    }
    if (lane == 0 && taken) atomicAdd(&s_count[E], taken);
#pragma unroll
    for (int i = 0; i < S; i++) s_sum[w][i * 32 + lane] = acc[i];
    if (lane == 0) s_sum[w][32 * S] = z;
    __syncthreads();
    for (int e = threadIdx.x; e <= E; e += kWarps * 32) {
        float v = 0.0f;
        for (int u = 0; u < kWarps; u++) v += s_sum[u][e < E ? e : 32 * S];
        part_counts[(int64_t)blockIdx.x * (E + 1) + e] = s_count[e];
        part_sums[(int64_t)blockIdx.x * (E + 1) + e] = v;
    }
}

// Partial results of each rank's slices, added in slice order.
__global__ void __launch_bounds__(128) router_reduce_kernel(const int2* ranks, int E, const int32_t* part_counts,
                                                           const float* part_sums, int32_t* counts, float* sums) {
    pdl_wait();
    const int e = blockIdx.x * 128 + threadIdx.x;
    if (e > E) return;
    const int2 r = ranks[blockIdx.y];  // first slice, number of slices
    int32_t c = 0;
    float v = 0.0f;
#pragma unroll 8
    for (int i = 0; i < r.y; i++) {
        c += part_counts[(int64_t)(r.x + i) * (E + 1) + e];
        v += part_sums[(int64_t)(r.x + i) * (E + 1) + e];
    }
    counts[(int64_t)blockIdx.y * (E + 1) + e] = c;
    sums[(int64_t)blockIdx.y * (E + 1) + e] = v;
}

// Sum over the gathered blocks of one expert's count, or (e = E) of the tokens that take part.
__device__ __forceinline__ int64_t gathered_count(const int32_t* gathered, int G, int E, int e) {
    int64_t c = 0;
#pragma unroll 4
    for (int g = 0; g < G; g++) c += gathered[(int64_t)g * (E + 1) + e];
    return c;
}

__global__ void __launch_bounds__(256) router_balance_kernel(const int32_t* gathered, int G, int E, int k,
                                                            const float* sums, float alpha, float beta, float* loss) {
    __shared__ float s[8];
    pdl_wait();
    gathered += (int64_t)blockIdx.x * G * (E + 1);
    sums += (int64_t)blockIdx.x * (E + 1);
    const int64_t n = gathered_count(gathered, G, E, E);
    const float number = (float)(n > 0 ? n : 1);
    float v = 0.0f;
    for (int e = threadIdx.x; e < E; e += 256)
        v += (float)gathered_count(gathered, G, E, e) / (number * k) * sums[e];
    v = warp_sum(v);
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 8; i++) v += s[i];
        loss[blockIdx.x] = alpha * E / number * v + beta / number * sums[E];
    }
}

template <typename T, int S>
__global__ void __launch_bounds__(kWarps * 32) router_backward_kernel(const Slice* slices, const T* logits, int64_t ld,
                                                                     const uint8_t* mask, int E, int k, int renormalize,
                                                                     const int32_t* indices, const float* weights,
                                                                     const float* lse_in, const int32_t* gathered,
                                                                     int G, const float* dweights, float alpha,
                                                                     float beta, const float* dloss, T* dlogits,
                                                                     int64_t dld) {
    __shared__ float s_extra[kWarps][32 * S];
    pdl_wait();
    const Slice sl = slices[blockIdx.x];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    gathered += (int64_t)sl.rank * G * (E + 1);
    const int64_t n = gathered_count(gathered, G, E, E);
    const float number = (float)(n > 0 ? n : 1), scale = dloss ? *dloss : 1.0f;
    const float ca = scale * alpha * E / number, cb = scale * 2.0f * beta / number;
    float f[S];
#pragma unroll
    for (int i = 0; i < S; i++) {
        const int e = i * 32 + lane;
        f[i] = e < E ? (float)gathered_count(gathered, G, E, e) / (number * k) : 0.0f;
        s_extra[w][e] = 0.0f;
    }
    __syncwarp();
    for (int t = w; t < sl.rows; t += kWarps) {
        const int64_t row = (int64_t)sl.row0 + t;
        const float lse = lse_in[row];
        int at = -1;
        float wgt = 0.0f, dw = 0.0f;
        if (lane < k) {
            at = indices[row * k + lane];
            wgt = weights[row * k + lane];
            if (dweights) dw = dweights[row * k + lane];
        }
        if (at < 0 || at >= E) at = -1, dw = 0.0f;
        // a token without a chosen expert takes part only through NaN logits
        bool on = !mask || mask[row] != 0;
        float l[S], p[S], inner = 0.0f;
        bool any = false;
#pragma unroll
        for (int i = 0; i < S; i++) {
            const int e = i * 32 + lane;
            l[i] = on && e < E ? to_float(logits[row * ld + e]) : -INFINITY;
            any |= !(l[i] == -INFINITY);
        }
        on = __any_sync(kAllLanes, any);
#pragma unroll
        for (int i = 0; i < S; i++) {
            p[i] = on && i * 32 + lane < E ? expf(l[i] - lse) : 0.0f;
            inner += p[i] * f[i];
        }
        inner = warp_sum(inner);
        const float dwsum = warp_sum(dw * wgt);
        if (at >= 0) s_extra[w][at] = wgt * (renormalize ? dw - dwsum : dw);
        __syncwarp();
        const float common = cb * lse - ca * inner - (renormalize ? 0.0f : dwsum);
#pragma unroll
        for (int i = 0; i < S; i++) {
            const int e = i * 32 + lane;
            if (e < E)
                dlogits[row * dld + e] = from_float<T>(on ? p[i] * (ca * f[i] + common) + s_extra[w][e] : 0.0f);
        }
        __syncwarp();
        if (at >= 0) s_extra[w][at] = 0.0f;
        __syncwarp();
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

template <typename T, typename F>
int by_experts(int E, F f) {
    if (E <= 64) return f.template operator()<T, 2>();
    if (E <= 128) return f.template operator()<T, 4>();
    if (E <= 256) return f.template operator()<T, 8>();
    if (E <= 512) return f.template operator()<T, 16>();
    return f.template operator()<T, 32>();
}
template <typename F>
int by_type(int dtype, int E, F f) {
    switch (dtype) {
        case SPARBIT_F32: return by_experts<float>(E, f);
        case SPARBIT_BF16: return by_experts<__nv_bfloat16>(E, f);
        default: return by_experts<__half>(E, f);
    }
}

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
        each = round_up(each ? each : 1, kWarps);
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
    if (!p || !counts || !sums || ld < (size_t)p->E) return SPARBIT_ERR_ARG;
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
        const int rc = by_type(p->dtype, p->E, [&]<typename T, int S>() {
            CU(launch(router_forward_kernel<T, S>, dim3((unsigned)p->slices.size()), dim3(kWarps * 32), 0, st,
                      (const Slice*)p->work, (const T*)logits, (int64_t)ld, mask, p->E, p->k, p->renormalize, indices,
                      weights, lse, pc, ps));
            return (int)SPARBIT_OK;
        });
        if (rc != SPARBIT_OK) return rc;
    }
    CU(launch(router_reduce_kernel, dim3((unsigned)(p->E / 128 + 1), (unsigned)p->n_ranks), dim3(128), 0, st,
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
    if (!p || !gathered || G < 1 || ld < (size_t)p->E || dlogits_ld < (size_t)p->E) return SPARBIT_ERR_ARG;
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
    return by_type(p->dtype, p->E, [&]<typename T, int S>() {
        CU(launch(router_backward_kernel<T, S>, dim3((unsigned)p->slices.size()), dim3(kWarps * 32), 0,
                  (cudaStream_t)stream, (const Slice*)p->work, (const T*)logits, (int64_t)ld, mask, p->E, p->k,
                  p->renormalize, indices, weights, lse, gathered, G, dweights, alpha, beta, dloss, (T*)dlogits,
                  (int64_t)dlogits_ld));
        return (int)SPARBIT_OK;
    });
}

}  // extern "C"
