// The norm of all gradients and their clipping: sums of squares in 64 bits for each rank's tensors, and, once the
// ranks' sums are gathered, every element times min(1, most / (norm + eps)).
//
// Bytes are the floor: all elements read, read again and written.  The tensors are cut into chunks; every CTA has a
// run of neighbouring chunks of about the same number of elements as the others'.  The second pass goes through each
// run backwards, so that what the first read last is found in L2.  Runs for four CTAs an SM, of which the sums' 56 registers
// let all be there together and the scaling's 92 two: eight, a chunk or two each, took 37 us in place of 34 for 43 MB.
// 475 MB of bf16 and f32 in 200 tensors: 83 us for the sums (5.7 TB/s; squares in 64 bits cost 2 of them), 172 for the
// scaling (5.5); of the whole 266, the rest is the gathered sums' kernel and the starts of the others.
#include <math.h>

#include <algorithm>
#include <new>
#include <utility>
#include <vector>

#include "train_common.cuh"

using namespace spb;

namespace {

constexpr int kChunkElements = 16384, kThreads = 256;
constexpr int kMostCtas = 148 * 4;

struct alignas(16) Tensor {
    const void* in;
    void* out;
    int64_t len;
    int32_t type, rank;
};
struct alignas(8) Chunk {
    int32_t tensor, index;  // chunk `index` of it
};

struct ClipArgs {
    const Tensor* tensors;
    const Chunk* chunks;        // by rank
    const int32_t* cta_begin;   // [CTAs + 1], chunks
    const int32_t* rank_parts;  // [ranks][2], parts
    double* parts;              // part of rank r from CTA b at [b + r]: runs meet every rank from left to right
    unsigned* control;          // ticket of the sums; whether the tensors that are set have outputs
    int n_ranks;
    double* sums;
    const double* gathered;
    int G;
    float most, eps;
    float* norms;
};

__device__ __forceinline__ double block_sum(double v, double* sm) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(kAllLanes, v, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = v;
    __syncthreads();
    v = sm[0];
    for (int i = 1; i < kThreads / 32; i++) v += sm[i];
    return v;
}

constexpr int kAhead = 4;  // accesses of a thread that are on their way together

template <typename T>
__device__ __forceinline__ double chunk_squares(const T* p, int n) {
    constexpr int A = 16 / sizeof(T);
    constexpr int kChains = 4;  // of additions that do not wait for one another
    double sum[kChains] = {};
    // squares are exact in 64 bits, of 32-bit numbers too
    auto square = [&](T x, int chain) {
        const double v = (double)to_float(x);
        sum[chain] = fma(v, v, sum[chain]);
    };
    const int head = min(n, (int)((16 - (uintptr_t)p % 16) % 16 / sizeof(T))), whole = (n - head) / A;
    const int done = head + whole * A;
    // the elements in front of the first whole access and behind the last
    if ((int)threadIdx.x < head) square(p[threadIdx.x], 0);
    if ((int)threadIdx.x < n - done) square(p[done + threadIdx.x], 1);
    const uint4* const v = reinterpret_cast<const uint4*>(p + head);
    uint4 k[2][kAhead];
    auto fetch = [&](int i0, uint4 (&to)[kAhead]) {
#pragma unroll
        for (int y = 0; y < kAhead; y++) {
            to[y] = make_uint4(0u, 0u, 0u, 0u);
            if (i0 + y * kThreads < whole) to[y] = v[i0 + y * kThreads];
        }
    };
    auto add = [&](const uint4 (&from)[kAhead]) {
#pragma unroll
        for (int y = 0; y < kAhead; y++) {
            const Pack<T, A> q = reinterpret_cast<const Pack<T, A>&>(from[y]);
#pragma unroll
            for (int i = 0; i < A; i++) square(q.v[i], i % kChains);
        }
    };
    fetch(threadIdx.x, k[0]);
    for (int i0 = threadIdx.x; i0 < whole; i0 += 2 * kThreads * kAhead) {
        fetch(i0 + kThreads * kAhead, k[1]);
        add(k[0]);
        fetch(i0 + 2 * kThreads * kAhead, k[0]);
        add(k[1]);
    }
    return (sum[0] + sum[1]) + (sum[2] + sum[3]);
}

__global__ void __launch_bounds__(kThreads) clip_sums_kernel(const __grid_constant__ ClipArgs g) {
    __shared__ double sm[kThreads / 32];
    __shared__ unsigned last;
    pdl_wait();
    pdl_trigger();
    const int lo = g.cta_begin[blockIdx.x], hi = g.cta_begin[blockIdx.x + 1];
    double sum = 0.0;
    int rank = -1;
    Chunk k = {};
    Tensor t = {};
    if (lo < hi) k = g.chunks[lo], t = g.tensors[k.tensor];
    for (int c = lo; c < hi; c++) {
        if (t.rank != rank) {
            if (rank >= 0) {
                sum = block_sum(sum, sm);
                if (threadIdx.x == 0) g.parts[blockIdx.x + rank] = sum;
                sum = 0.0;
            }
            rank = t.rank;
        }
        const int64_t at = (int64_t)k.index * kChunkElements;
        const int n = (int)min((int64_t)kChunkElements, t.len - at);
        if (t.type == SPARBIT_F32) sum += chunk_squares((const float*)t.in + at, n);
        else if (t.type == SPARBIT_BF16) sum += chunk_squares((const __nv_bfloat16*)t.in + at, n);
        else sum += chunk_squares((const __half*)t.in + at, n);
        if (c + 1 < hi) k = g.chunks[c + 1], t = g.tensors[k.tensor];
    }
    if (rank >= 0) {
        sum = block_sum(sum, sm);
        if (threadIdx.x == 0) g.parts[blockIdx.x + rank] = sum;
    }
    // the CTA that comes last adds the parts, always in the same order
    if (threadIdx.x == 0) {
        __threadfence();
        last = atomicAdd(g.control, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int r = warp; r < g.n_ranks; r += kThreads / 32) {
        // runs are in order, so that a rank's parts lie side by side
        const int lo_part = g.rank_parts[2 * r], hi_part = g.rank_parts[2 * r + 1];
        double s = 0.0;
#pragma unroll 8
        for (int i = lo_part + lane; i < hi_part; i += 32) s += __ldcg(g.parts + i);
#pragma unroll
        for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(kAllLanes, s, o);
        if (lane == 0) g.sums[r] = s;
    }
    if (threadIdx.x == 0) g.control[0] = 0;
}

template <typename T>
__device__ __forceinline__ void scale_chunk(const T* in, T* out, int n, float by) {
    constexpr int A = 16 / sizeof(T);
    if (((uintptr_t)in ^ (uintptr_t)out) % 16) {
        for (int i = threadIdx.x; i < n; i += kThreads) out[i] = from_float<T>(to_float(in[i]) * by);
        return;
    }
    const int head = min(n, (int)((16 - (uintptr_t)in % 16) % 16 / sizeof(T))), whole = (n - head) / A;
    if ((int)threadIdx.x < head) out[threadIdx.x] = from_float<T>(to_float(in[threadIdx.x]) * by);
    const uint4* const from = reinterpret_cast<const uint4*>(in + head);
    uint4* const to = reinterpret_cast<uint4*>(out + head);
    for (int i0 = threadIdx.x; i0 < whole; i0 += kThreads * kAhead) {
        uint4 k[kAhead];
#pragma unroll
        for (int y = 0; y < kAhead; y++)
            if (i0 + y * kThreads < whole) k[y] = from[i0 + y * kThreads];
#pragma unroll
        for (int y = 0; y < kAhead; y++) {
            if (i0 + y * kThreads >= whole) break;
            Pack<T, A> q = reinterpret_cast<const Pack<T, A>&>(k[y]);
#pragma unroll
            for (int i = 0; i < A; i++) q.v[i] = from_float<T>(to_float(q.v[i]) * by);
            to[i0 + y * kThreads] = reinterpret_cast<const uint4&>(q);
        }
    }
    const int done = head + whole * A;
    if ((int)threadIdx.x < n - done) out[done + threadIdx.x] = from_float<T>(to_float(in[done + threadIdx.x]) * by);
}

__device__ __forceinline__ void factor_of(const ClipArgs& g, int rank, double* sm, float& norm, float& factor) {
    double s = 0.0;
    for (int i = threadIdx.x; i < g.G; i += kThreads) s += g.gathered[(int64_t)rank * g.G + i];
    s = sqrt(block_sum(s, sm));
    norm = (float)s;
    // a NaN stays one; 0 / 0 (nothing allowed of nothing) is 1
    const double f = (double)g.most / (s + (double)g.eps);
    factor = s == 0.0 ? 1.0f : f < 1.0 ? (float)f : s != s ? (float)s : 1.0f;
}

__global__ void __launch_bounds__(kThreads) clip_scale_kernel(const __grid_constant__ ClipArgs g) {
    __shared__ double sm[kThreads / 32];
    pdl_wait();
    pdl_trigger();
    // not an argument: a captured call follows what is set when it is replayed
    const bool write = g.control[1] != 0;
    float norm, factor = 1.0f;
    for (int r = blockIdx.x; r < g.n_ranks; r += gridDim.x) {
        factor_of(g, r, sm, norm, factor);
        if (threadIdx.x == 0) g.norms[2 * r] = norm, g.norms[2 * r + 1] = factor;
    }
    if (!write) return;
    const int lo = g.cta_begin[blockIdx.x], hi = g.cta_begin[blockIdx.x + 1];
    int rank = -1;
    for (int c = hi - 1; c >= lo; c--) {
        const Chunk k = g.chunks[c];
        const Tensor t = g.tensors[k.tensor];
        if (t.rank != rank) {
            rank = t.rank;
            factor_of(g, rank, sm, norm, factor);
        }
        if (factor == 1.0f && t.in == t.out) continue;
        const int64_t at = (int64_t)k.index * kChunkElements;
        const int n = (int)min((int64_t)kChunkElements, t.len - at);
        if (t.type == SPARBIT_F32) scale_chunk((const float*)t.in + at, (float*)t.out + at, n, factor);
        else if (t.type == SPARBIT_BF16) scale_chunk((const __nv_bfloat16*)t.in + at, (__nv_bfloat16*)t.out + at, n, factor);
        else scale_chunk((const __half*)t.in + at, (__half*)t.out + at, n, factor);
    }
}

// Address ranges, for the question whether another one meets any of them.
struct Ranges {
    std::vector<std::pair<uintptr_t, uintptr_t>> v;  // by their first bytes; second: how far this one and those before it reach
    void finish() {
        std::sort(v.begin(), v.end());
        for (size_t i = 1; i < v.size(); i++) v[i].second = std::max(v[i].second, v[i - 1].second);
    }
    bool meet(const void* p, size_t bytes) const {
        const uintptr_t lo = (uintptr_t)p;
        const auto behind = std::lower_bound(v.begin(), v.end(), std::pair<uintptr_t, uintptr_t>(lo + bytes, 0));
        return behind != v.begin() && (behind - 1)->second > lo;
    }
};

}  // namespace

struct sparbit_clip_plan_s {
    int n_ranks = 0, ctas = 0;
    std::vector<Tensor> tensors;
    std::vector<Chunk> chunks;
    std::vector<int32_t> cta_begin, rank_parts;
    Ranges inputs, outputs;  // of the tensors that are set
    char* work = nullptr;
    int device = -1;
    bool set = false;
    unsigned write = 0;  // as it stands in the workspace

    size_t off_tensors() const { return 256; }
    size_t off_chunks() const { return off_tensors() + round_up(tensors.size() * sizeof(Tensor), 256); }
    size_t off_ctas() const { return off_chunks() + round_up(chunks.size() * sizeof(Chunk), 256); }
    size_t off_ranks() const { return off_ctas() + round_up(cta_begin.size() * sizeof(int32_t), 256); }
    size_t off_parts() const { return off_ranks() + round_up(rank_parts.size() * sizeof(int32_t), 256); }
    size_t work_bytes() const { return off_parts() + (size_t)(ctas + n_ranks) * sizeof(double); }
};

namespace {

using Plan = sparbit_clip_plan_s;

int ready(const Plan* p) {
    if (!p->work || !p->set) return SPARBIT_ERR_WORKSPACE;
    int cur = -1;
    CU(cudaGetDevice(&cur));
    return cur == p->device ? SPARBIT_OK : SPARBIT_ERR_ARG;
}

ClipArgs common_args(const Plan* p) {
    ClipArgs g = {};
    g.tensors = (const Tensor*)(p->work + p->off_tensors());
    g.chunks = (const Chunk*)(p->work + p->off_chunks());
    g.cta_begin = (const int32_t*)(p->work + p->off_ctas());
    g.rank_parts = (const int32_t*)(p->work + p->off_ranks());
    g.parts = (double*)(p->work + p->off_parts());
    g.control = (unsigned*)p->work;
    g.n_ranks = p->n_ranks;
    return g;
}

}  // namespace

extern "C" {

int sparbit_clip_plan_create(int n_ranks, size_t n, const size_t* lengths, const int* dtypes, const int* ranks,
                             sparbit_clip_plan_t** out) {
    if (!out) return SPARBIT_ERR_ARG;
    *out = nullptr;
    if (n_ranks < 1 || n < 1 || !lengths || !dtypes) return SPARBIT_ERR_ARG;
    if (n_ranks > 65535 || n > (1u << 24)) return SPARBIT_ERR_LIMIT;
    size_t all = 0, pieces = 0;
    for (size_t i = 0; i < n; i++) {
        if (!known_dtype(dtypes[i]) || (ranks && (ranks[i] < 0 || ranks[i] >= n_ranks))) return SPARBIT_ERR_ARG;
        if (lengths[i] > kMostElements - all) return SPARBIT_ERR_OVERFLOW;
        all += lengths[i];
        pieces += (lengths[i] + kChunkElements - 1) / kChunkElements;
        if (pieces > 0x7fffffffu) return SPARBIT_ERR_LIMIT;
    }
    Plan* p = new (std::nothrow) Plan();
    if (!p) return SPARBIT_ERR_NOMEM;
    try {
        p->n_ranks = n_ranks;
        std::vector<int32_t> order(n);
        for (size_t i = 0; i < n; i++) {
            order[i] = (int32_t)i;
            p->tensors.push_back(Tensor{nullptr, nullptr, (int64_t)lengths[i], dtypes[i], ranks ? ranks[i] : 0});
        }
        std::stable_sort(order.begin(), order.end(),
                         [&](int32_t a, int32_t b) { return p->tensors[a].rank < p->tensors[b].rank; });
        std::vector<int32_t> begin((size_t)n_ranks + 1, 0);  // of each rank's chunks
        // about as many bytes for every CTA; a chunk counts for some more than it has
        std::vector<double> upto{0.0};
        for (int32_t i : order) {
            const Tensor& t = p->tensors[i];
            const int32_t each = (int32_t)((t.len + kChunkElements - 1) / kChunkElements);
            for (int32_t j = 0; j < each; j++) {
                p->chunks.push_back(Chunk{i, j});
                const double here = (double)std::min<int64_t>(kChunkElements, t.len - (int64_t)j * kChunkElements);
                upto.push_back(upto.back() + here * (double)elem_size(t.type) + 2048.0);
            }
            begin[t.rank + 1] += each;
        }
        for (int r = 0; r < n_ranks; r++) begin[r + 1] += begin[r];
        p->ctas = (int)std::max<size_t>(1, std::min<size_t>(kMostCtas, p->chunks.size()));
        for (int b = 0; b <= p->ctas; b++) {
            const double until = upto.back() * b / p->ctas;
            // the chunk whose middle lies behind the boundary begins the next run
            const size_t at = std::lower_bound(upto.begin(), upto.end(), until) - upto.begin();
            size_t cut = at;
            if (at > 0 && at < upto.size() && until - upto[at - 1] < upto[at] - until) cut = at - 1;
            p->cta_begin.push_back(b == p->ctas ? (int32_t)p->chunks.size() : (int32_t)std::min(cut, p->chunks.size()));
        }
        p->cta_begin[0] = 0;
        // the CTA that holds a chunk: the last whose run begins at it or before it
        auto holder = [&](int32_t chunk) {
            return (int32_t)(std::upper_bound(p->cta_begin.begin(), p->cta_begin.end() - 1, chunk) - p->cta_begin.begin()) - 1;
        };
        for (int r = 0; r < n_ranks; r++) {
            const bool any = begin[r] < begin[r + 1];
            p->rank_parts.push_back(any ? holder(begin[r]) + r : 0);
            p->rank_parts.push_back(any ? holder(begin[r + 1] - 1) + r + 1 : 0);
        }
    } catch (const std::bad_alloc&) {
        delete p;
        return SPARBIT_ERR_NOMEM;
    }
    *out = p;
    return SPARBIT_OK;
}

int sparbit_clip_plan_destroy(sparbit_clip_plan_t* p) {
    delete p;
    return SPARBIT_OK;
}

size_t sparbit_clip_plan_workspace_bytes(const sparbit_clip_plan_t* p) { return p ? p->work_bytes() : 0; }

int sparbit_clip_plan_set_workspace(sparbit_clip_plan_t* p, void* dev, size_t bytes) {
    if (!p) return SPARBIT_ERR_ARG;
    if (!dev || bytes < p->work_bytes() || (uintptr_t)dev % 16) return SPARBIT_ERR_WORKSPACE;
    p->work = nullptr;
    p->set = false;
    p->write = 0;
    CU(cudaGetDevice(&p->device));
    char* base = (char*)dev;
    CU(cudaMemset(base, 0, 256));
    if (!p->chunks.empty())
        CU(cudaMemcpy(base + p->off_chunks(), p->chunks.data(), p->chunks.size() * sizeof(Chunk), cudaMemcpyHostToDevice));
    CU(cudaMemcpy(base + p->off_ctas(), p->cta_begin.data(), p->cta_begin.size() * sizeof(int32_t), cudaMemcpyHostToDevice));
    CU(cudaMemcpy(base + p->off_ranks(), p->rank_parts.data(), p->rank_parts.size() * sizeof(int32_t), cudaMemcpyHostToDevice));
    CU(cudaMemset(base + p->off_parts(), 0, (size_t)(p->ctas + p->n_ranks) * sizeof(double)));
    CU(cudaDeviceSynchronize());
    p->work = base;
    return SPARBIT_OK;
}

int sparbit_clip_plan_set_tensors(sparbit_clip_plan_t* p, const void* const* in, void* const* out) {
    if (!p || !in) return SPARBIT_ERR_ARG;
    const size_t n = p->tensors.size();
    Ranges inputs, outputs;
    try {
        struct Span {
            uintptr_t lo, hi;
            bool written;
        };
        std::vector<Span> spans;
        for (size_t i = 0; i < n; i++) {
            const Tensor& t = p->tensors[i];
            if (!t.len) continue;
            const size_t es = elem_size(t.type);
            if (!in[i] || (uintptr_t)in[i] % es || (out && (!out[i] || (uintptr_t)out[i] % es))) return SPARBIT_ERR_ARG;
            const uintptr_t a = (uintptr_t)in[i], b = out ? (uintptr_t)out[i] : 0, bytes = (uintptr_t)t.len * es;
            if (a + bytes < a || (out && b + bytes < b)) return SPARBIT_ERR_ARG;
            inputs.v.emplace_back(a, a + bytes);
            if (out) outputs.v.emplace_back(b, b + bytes);
            if (out) spans.push_back(Span{b, b + bytes, true});
            if (!out || a != b) spans.push_back(Span{a, a + bytes, false});
        }
        if (p->work && out) spans.push_back(Span{(uintptr_t)p->work, (uintptr_t)p->work + p->work_bytes(), false});
        std::sort(spans.begin(), spans.end(), [](const Span& x, const Span& y) { return x.lo < y.lo; });
        uintptr_t any = 0, written = 0;  // how far those before reach
        for (const Span& s : spans) {
            if (s.lo < (s.written ? any : written)) return SPARBIT_ERR_ALIAS;
            any = std::max(any, s.hi);
            if (s.written) written = std::max(written, s.hi);
        }
        inputs.finish(), outputs.finish();
    } catch (const std::bad_alloc&) {
        return SPARBIT_ERR_NOMEM;
    }
    if (!p->work) return SPARBIT_ERR_WORKSPACE;
    int cur = -1;
    CU(cudaGetDevice(&cur));
    if (cur != p->device) return SPARBIT_ERR_ARG;
    p->set = false;
    for (size_t i = 0; i < n; i++) p->tensors[i].in = in[i], p->tensors[i].out = out ? out[i] : nullptr;
    CU(cudaDeviceSynchronize());
    CU(cudaMemcpy(p->work + p->off_tensors(), p->tensors.data(), n * sizeof(Tensor), cudaMemcpyHostToDevice));
    const unsigned write = out != nullptr;
    if (write != p->write) CU(cudaMemcpy(p->work + sizeof write, &write, sizeof write, cudaMemcpyHostToDevice));
    p->write = write;
    CU(cudaDeviceSynchronize());
    p->inputs = std::move(inputs), p->outputs = std::move(outputs);
    p->set = true;
    return SPARBIT_OK;
}

int sparbit_clip_sums(sparbit_clip_plan_t* p, double* sums, void* stream) {
    if (!p || !sums) return SPARBIT_ERR_ARG;
    if (regions_overlap({sums, 1, (size_t)p->n_ranks * 8, 0}, {p->work, 1, p->work_bytes(), 0})) return SPARBIT_ERR_ALIAS;
    if (misaligned(8, {sums})) return SPARBIT_ERR_ARG;
    const int e = ready(p);
    if (e != SPARBIT_OK) return e;
    if (p->inputs.meet(sums, (size_t)p->n_ranks * 8)) return SPARBIT_ERR_ALIAS;
    ClipArgs g = common_args(p);
    g.sums = sums;
    CU(launch(clip_sums_kernel, dim3(p->ctas), dim3(kThreads), 0, (cudaStream_t)stream, g));
    return SPARBIT_OK;
}

int sparbit_clip_scale(sparbit_clip_plan_t* p, const double* gathered, int G, float most, float eps, float* norms,
                       void* stream) {
    if (!p || !gathered || !norms || G < 1 || !(most >= 0.0f) || !(eps >= 0.0f) || !isfinite(eps)) return SPARBIT_ERR_ARG;
    const Region rg{gathered, 1, (size_t)p->n_ranks * G * 8, 0}, rn{norms, 1, (size_t)p->n_ranks * 8, 0};
    if (regions_overlap(rn, rg) || regions_overlap(rn, {p->work, 1, p->work_bytes(), 0})) return SPARBIT_ERR_ALIAS;
    if (misaligned(8, {gathered}) || misaligned(4, {norms})) return SPARBIT_ERR_ARG;
    const int e = ready(p);
    if (e != SPARBIT_OK) return e;
    if (p->inputs.meet(norms, rn.width) || p->outputs.meet(norms, rn.width) || p->outputs.meet(gathered, rg.width))
        return SPARBIT_ERR_ALIAS;
    ClipArgs g = common_args(p);
    g.gathered = gathered, g.G = G, g.most = most, g.eps = eps, g.norms = norms;
    CU(launch(clip_scale_kernel, dim3(p->ctas), dim3(kThreads), 0, (cudaStream_t)stream, g));
    return SPARBIT_OK;
}

}  // extern "C"
