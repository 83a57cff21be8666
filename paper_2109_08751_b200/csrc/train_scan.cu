// Gated linear recurrence: h_t = a_t h_{t-1} + (1 - a_t) x_t, a = sigmoid(gate), per channel.
//
// A sequence is cut into pieces of kPiece steps.  What a piece does to the state that enters it is
// the pair (A, H): h -> A h + H, with A the product of its a_t; pairs compose, which is what lets
// the pieces be worked on side by side.
#include <new>
#include <vector>

#include "train_common.cuh"

using namespace spb;

namespace {

constexpr int kPiece = 128;        // steps of a piece
constexpr int kFwdWarps = 8;       // 16 steps a warp
constexpr int kBwdWarps = 16;      // 8 steps a warp: three inputs are held in registers

struct Piece {
    int64_t row0;
    int32_t seq;
    int32_t len;
};
struct Seq {
    int32_t first, pieces;  // into the list of pieces
};

// a = 1/(1+exp(-g)) and 1 - a, neither of them by cancellation
__device__ __forceinline__ void gate_pair(float g, float& a, float& keep) {
    const float t = __expf(-fabsf(g));
    const float r = __fdividef(1.0f, 1.0f + t);
    const float u = t * r;
    a = g >= 0.0f ? r : u;
    keep = g >= 0.0f ? u : r;
    if (g != g) a = keep = g;
}

template <typename T, int V>
__device__ __forceinline__ void load_row(const T* p, int64_t row, int64_t ld, int channel, bool on, float (&out)[V]) {
    Pack<T, V> v;
    if (on) v = *reinterpret_cast<const Pack<T, V>*>(p + row * ld + channel);
#pragma unroll
    for (int i = 0; i < V; i++) out[i] = on ? to_float(v.v[i]) : 0.0f;
}
template <typename T, int V>
__device__ __forceinline__ void store_row(T* p, int64_t row, int64_t ld, int channel, const float (&in)[V]) {
    Pack<T, V> v;
#pragma unroll
    for (int i = 0; i < V; i++) v.v[i] = from_float<T>(in[i]);
    *reinterpret_cast<Pack<T, V>*>(p + row * ld + channel) = v;
}

// What each piece does to a state (kReverse: to a gradient), pairs[piece][2][D].
template <typename T, int V, bool kReverse>
__global__ void __launch_bounds__(kFwdWarps * 32) scan_pairs_kernel(const Piece* pieces, const T* gate, int64_t gate_ld,
                                                                   const T* in, int64_t in_ld, int D, float* pairs) {
    constexpr int R = kPiece / kFwdWarps;
    __shared__ float sA[kFwdWarps][32 * V], sH[kFwdWarps][32 * V];
    pdl_wait();
    const Piece pc = pieces[blockIdx.x];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int ch = (blockIdx.y * 32 + lane) * V;
    float A[V], H[V];
#pragma unroll
    for (int i = 0; i < V; i++) A[i] = 1.0f, H[i] = 0.0f;
#pragma unroll 4
    for (int j = 0; j < R; j++) {
        const int t = kReverse ? w * R + R - 1 - j : w * R + j;
        const bool on = t < pc.len && ch < D;
        float g[V], x[V];
        load_row<T, V>(gate, pc.row0 + t, gate_ld, ch, on, g);
        load_row<T, V>(in, pc.row0 + t, in_ld, ch, on, x);
        if (!on) continue;
#pragma unroll
        for (int i = 0; i < V; i++) {
            float a, keep;
            gate_pair(g[i], a, keep);
            H[i] = kReverse ? a * (H[i] + x[i]) : a * H[i] + keep * x[i];
            A[i] *= a;
        }
    }
#pragma unroll
    for (int i = 0; i < V; i++) sA[w][lane * V + i] = A[i], sH[w][lane * V + i] = H[i];
    __syncthreads();
    if (w == 0 && ch < D) {
        float a[V], h[V];
#pragma unroll
        for (int i = 0; i < V; i++) a[i] = 1.0f, h[i] = 0.0f;
        for (int q = 0; q < kFwdWarps; q++) {
            const int u = kReverse ? kFwdWarps - 1 - q : q;
#pragma unroll
            for (int i = 0; i < V; i++) {
                h[i] = sA[u][lane * V + i] * h[i] + sH[u][lane * V + i];
                a[i] *= sA[u][lane * V + i];
            }
        }
        store_row<float, V>(pairs, (int64_t)blockIdx.x * 2, D, ch, a);
        store_row<float, V>(pairs, (int64_t)blockIdx.x * 2 + 1, D, ch, h);
    }
}

// The state that enters each piece, and each sequence's summary.
template <bool kReverse>
__global__ void __launch_bounds__(128) scan_carry_kernel(const Seq* seqs, const float* pairs, const float* first,
                                                        int64_t first_ld, int D, float* carry, float* summary) {
    pdl_wait();
    const int ch = blockIdx.x * 128 + threadIdx.x;
    if (ch >= D) return;
    const Seq s = seqs[blockIdx.y];
    float h = first ? first[blockIdx.y * first_ld + ch] : 0.0f, total = 1.0f;
#pragma unroll 8
    for (int j = 0; j < s.pieces; j++) {
        const int64_t c = s.first + (kReverse ? s.pieces - 1 - j : j);
        const float a = pairs[c * 2 * D + ch], b = pairs[(c * 2 + 1) * D + ch];
        carry[c * D + ch] = h;
        h = a * h + b;
        total *= a;
    }
    if (summary) {
        summary[(int64_t)blockIdx.y * 2 * D + ch] = total;
        summary[((int64_t)blockIdx.y * 2 + 1) * D + ch] = h;
    }
}

// The states of a piece from the state that enters it.
template <typename T, int V>
__global__ void __launch_bounds__(kFwdWarps * 32) scan_forward_kernel(const Piece* pieces, const T* gate,
                                                                     int64_t gate_ld, const T* x, int64_t x_ld, int D,
                                                                     const float* carry, T* y, int64_t y_ld) {
    constexpr int R = kPiece / kFwdWarps;
    __shared__ float sA[kFwdWarps][32 * V], sH[kFwdWarps][32 * V];
    pdl_wait();
    const Piece pc = pieces[blockIdx.x];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int ch = (blockIdx.y * 32 + lane) * V;
    float a[R][V], b[R][V], A[V], H[V];
#pragma unroll
    for (int j = 0; j < R; j++) {
        const bool on = w * R + j < pc.len && ch < D;
        load_row<T, V>(gate, pc.row0 + w * R + j, gate_ld, ch, on, a[j]);
        load_row<T, V>(x, pc.row0 + w * R + j, x_ld, ch, on, b[j]);
    }
#pragma unroll
    for (int i = 0; i < V; i++) A[i] = 1.0f, H[i] = 0.0f;
#pragma unroll
    for (int j = 0; j < R; j++) {
        const bool on = w * R + j < pc.len;
#pragma unroll
        for (int i = 0; i < V; i++) {
            float keep;
            gate_pair(a[j][i], a[j][i], keep);
            b[j][i] *= keep;
            if (!on) a[j][i] = 1.0f, b[j][i] = 0.0f;
            H[i] = a[j][i] * H[i] + b[j][i];
            A[i] *= a[j][i];
        }
    }
#pragma unroll
    for (int i = 0; i < V; i++) sA[w][lane * V + i] = A[i], sH[w][lane * V + i] = H[i];
    __syncthreads();
    if (ch >= D) return;
    float h[V];
    load_row<float, V>(carry, blockIdx.x, D, ch, true, h);
    for (int u = 0; u < w; u++)
#pragma unroll
        for (int i = 0; i < V; i++) h[i] = sA[u][lane * V + i] * h[i] + sH[u][lane * V + i];
#pragma unroll
    for (int j = 0; j < R; j++) {
#pragma unroll
        for (int i = 0; i < V; i++) h[i] = a[j][i] * h[i] + b[j][i];
        if (w * R + j < pc.len) store_row<T, V>(y, pc.row0 + w * R + j, y_ld, ch, h);
    }
}

// The gradients of a piece, from the state that enters it at its start and the gradient that
// enters it at its end; its states are computed again.
template <typename T, int V>
__global__ void __launch_bounds__(kBwdWarps * 32) scan_backward_kernel(const Piece* pieces, const T* gate,
                                                                      int64_t gate_ld, const T* x, int64_t x_ld,
                                                                      const T* dy, int64_t dy_ld, int D,
                                                                      const float* carry, const float* back, T* dgate,
                                                                      int64_t dgate_ld, T* dx, int64_t dx_ld) {
    constexpr int R = kPiece / kBwdWarps;
    __shared__ float sA[kBwdWarps][32 * V], sH[kBwdWarps][32 * V], sG[kBwdWarps][32 * V];
    pdl_wait();
    const Piece pc = pieces[blockIdx.x];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int ch = (blockIdx.y * 32 + lane) * V;
    float gt[R][V], xv[R][V], d[R][V], A[V], H[V], G[V];
#pragma unroll
    for (int j = 0; j < R; j++) {
        const bool on = w * R + j < pc.len && ch < D;
        load_row<T, V>(gate, pc.row0 + w * R + j, gate_ld, ch, on, gt[j]);
        load_row<T, V>(x, pc.row0 + w * R + j, x_ld, ch, on, xv[j]);
        load_row<T, V>(dy, pc.row0 + w * R + j, dy_ld, ch, on, d[j]);
    }
#pragma unroll
    for (int i = 0; i < V; i++) A[i] = 1.0f, H[i] = 0.0f, G[i] = 0.0f;
#pragma unroll
    for (int j = 0; j < R; j++) {
        if (w * R + j >= pc.len) break;
#pragma unroll
        for (int i = 0; i < V; i++) {
            float a, keep;
            gate_pair(gt[j][i], a, keep);
            H[i] = a * H[i] + keep * xv[j][i];
            // the map of the gradient, built front to back: c -> G + A c with this step's dy seen
            // through all the steps before it
            A[i] *= a;
            G[i] += A[i] * d[j][i];
        }
    }
#pragma unroll
    for (int i = 0; i < V; i++)
        sA[w][lane * V + i] = A[i], sH[w][lane * V + i] = H[i], sG[w][lane * V + i] = G[i];
    __syncthreads();
    if (ch >= D) return;
    float h[R + 1][V], c[V];
    load_row<float, V>(carry, blockIdx.x, D, ch, true, h[0]);
    load_row<float, V>(back, blockIdx.x, D, ch, true, c);
    for (int u = 0; u < w; u++)
#pragma unroll
        for (int i = 0; i < V; i++) h[0][i] = sA[u][lane * V + i] * h[0][i] + sH[u][lane * V + i];
    for (int u = kBwdWarps - 1; u > w; u--)
#pragma unroll
        for (int i = 0; i < V; i++) c[i] = sA[u][lane * V + i] * c[i] + sG[u][lane * V + i];
#pragma unroll
    for (int j = 0; j < R; j++)
#pragma unroll
        for (int i = 0; i < V; i++) {
            float a, keep;
            gate_pair(gt[j][i], a, keep);
            h[j + 1][i] = a * h[j][i] + keep * xv[j][i];
        }
#pragma unroll
    for (int j = R - 1; j >= 0; j--) {
        if (w * R + j >= pc.len) continue;
        float dg[V], dxv[V];
#pragma unroll
        for (int i = 0; i < V; i++) {
            float a, keep;
            gate_pair(gt[j][i], a, keep);
            const float g = d[j][i] + c[i];
            dxv[i] = g * keep;
            dg[i] = dxv[i] * (h[j][i] - xv[j][i]) * a;
            c[i] = a * g;
        }
        store_row<T, V>(dgate, pc.row0 + w * R + j, dgate_ld, ch, dg);
        store_row<T, V>(dx, pc.row0 + w * R + j, dx_ld, ch, dxv);
    }
}

template <typename T, int V>
__global__ void __launch_bounds__(128) scan_step_kernel(const T* gate, int64_t gate_ld, const T* x, int64_t x_ld,
                                                       const int32_t* slots, int64_t n_slots, int D,
                                                       const float* state_in, float* state_out, int64_t state_ld, T* y,
                                                       int64_t y_ld) {
    pdl_wait();
    const int64_t row = blockIdx.x;
    const int ch = (blockIdx.y * 128 + threadIdx.x) * V;
    if (ch >= D) return;
    const int64_t slot = slots ? slots[row] : row;
    float g[V], v[V], h[V];
    load_row<T, V>(gate, row, gate_ld, ch, true, g);
    load_row<T, V>(x, row, x_ld, ch, true, v);
    const bool on = slot >= 0 && slot < n_slots;
    load_row<float, V>(state_in, on ? slot : 0, state_ld, ch, on, h);
#pragma unroll
    for (int i = 0; i < V; i++) {
        float a, keep;
        gate_pair(g[i], a, keep);
        h[i] = on ? a * h[i] + keep * v[i] : 0.0f;
    }
    if (on) store_row<float, V>(state_out, slot, state_ld, ch, h);
    store_row<T, V>(y, row, y_ld, ch, h);
}

__global__ void __launch_bounds__(128) scan_join_kernel(int P, int first_rank, int D, const float* gathered,
                                                       const float* h0, float* out, int64_t out_ld, int reverse) {
    pdl_wait();
    const int ch = blockIdx.x * 128 + threadIdx.x;
    if (ch >= D) return;
    const int r = first_rank + blockIdx.y;
    const float* blocks = gathered + (int64_t)blockIdx.y * P * 2 * D + ch;
    float h = h0 ? h0[ch] : 0.0f;
    const int n = reverse ? P - 1 - r : r;
#pragma unroll 4
    for (int j = 0; j < n; j++) {
        const int64_t k = reverse ? P - 1 - j : j;
        h = blocks[k * 2 * D] * h + blocks[(k * 2 + 1) * D];
    }
    out[blockIdx.y * out_ld + ch] = h;
}

}  // namespace

struct sparbit_scan_plan_s {
    int n_seqs = 0;
    int D = 0;
    int dtype = 0;
    size_t rows = 0;
    std::vector<Piece> pieces;
    std::vector<Seq> seqs;
    char* work = nullptr;
    int device = -1;

    size_t off_seqs() const { return round_up(pieces.size() * sizeof(Piece), 256); }
    size_t off_pairs() const { return off_seqs() + round_up(seqs.size() * sizeof(Seq), 256); }
    size_t off_carry() const { return off_pairs() + round_up(pieces.size() * 2 * D * sizeof(float), 256); }
    size_t off_back() const { return off_carry() + round_up(pieces.size() * D * sizeof(float), 256); }
    size_t work_bytes() const { return off_back(); }
};

namespace {

int ready(const sparbit_scan_plan_s* p) {
    if (!p->work) return SPARBIT_ERR_WORKSPACE;
    int cur = -1;
    CU(cudaGetDevice(&cur));
    return cur == p->device ? SPARBIT_OK : SPARBIT_ERR_ARG;
}

template <typename T, int V>
int run_forward(sparbit_scan_plan_s* p, const void* gate, size_t gate_ld, const void* x, size_t x_ld, const float* h0,
                size_t h0_ld, void* y, size_t y_ld, float* summary, float* carry, cudaStream_t st) {
    const Piece* pieces = (const Piece*)p->work;
    const Seq* seqs = (const Seq*)(p->work + p->off_seqs());
    float* pairs = (float*)(p->work + p->off_pairs());
    if (!carry) carry = (float*)(p->work + p->off_carry());
    const dim3 grid((unsigned)p->pieces.size(), (unsigned)((p->D + 32 * V - 1) / (32 * V)));
    if (grid.x)
        CU(launch(scan_pairs_kernel<T, V, false>, grid, dim3(kFwdWarps * 32), 0, st, pieces, (const T*)gate,
                  (int64_t)gate_ld, (const T*)x, (int64_t)x_ld, p->D, pairs));
    CU(launch(scan_carry_kernel<false>, dim3((p->D + 127) / 128, p->n_seqs), dim3(128), 0, st, seqs,
              (const float*)pairs, h0, (int64_t)h0_ld, p->D, carry, summary));
    if (y && grid.x)
        CU(launch(scan_forward_kernel<T, V>, grid, dim3(kFwdWarps * 32), 0, st, pieces, (const T*)gate,
                  (int64_t)gate_ld, (const T*)x, (int64_t)x_ld, p->D, (const float*)carry, (T*)y, (int64_t)y_ld));
    return SPARBIT_OK;
}

template <typename T, int V>
int run_backward(sparbit_scan_plan_s* p, const void* gate, size_t gate_ld, const void* x, size_t x_ld,
                 const float* carry, const void* dy, size_t dy_ld, const float* dlast, size_t dlast_ld, void* dgate,
                 size_t dgate_ld, void* dx, size_t dx_ld, float* dsummary, cudaStream_t st) {
    const Piece* pieces = (const Piece*)p->work;
    const Seq* seqs = (const Seq*)(p->work + p->off_seqs());
    float* pairs = (float*)(p->work + p->off_pairs());
    float* back = (float*)(p->work + p->off_carry());
    const dim3 grid((unsigned)p->pieces.size(), (unsigned)((p->D + 32 * V - 1) / (32 * V)));
    if (grid.x)
        CU(launch(scan_pairs_kernel<T, V, true>, grid, dim3(kFwdWarps * 32), 0, st, pieces, (const T*)gate,
                  (int64_t)gate_ld, (const T*)dy, (int64_t)dy_ld, p->D, pairs));
    CU(launch(scan_carry_kernel<true>, dim3((p->D + 127) / 128, p->n_seqs), dim3(128), 0, st, seqs,
              (const float*)pairs, dlast, (int64_t)dlast_ld, p->D, back, dsummary));
    if (dx && grid.x)
        CU(launch(scan_backward_kernel<T, V>, grid, dim3(kBwdWarps * 32), 0, st, pieces, (const T*)gate,
                  (int64_t)gate_ld, (const T*)x, (int64_t)x_ld, (const T*)dy, (int64_t)dy_ld, p->D, carry,
                  (const float*)back, (T*)dgate, (int64_t)dgate_ld, (T*)dx, (int64_t)dx_ld));
    return SPARBIT_OK;
}

// Calls f.template operator()<T, V>() for the plan's type and the number of channels a lane takes.
template <typename F>
int by_type(int dtype, int V, F f) {
    switch (dtype) {
        case SPARBIT_F32: return V == 2 ? f.template operator()<float, 2>() : f.template operator()<float, 1>();
        case SPARBIT_BF16:
            return V == 2 ? f.template operator()<__nv_bfloat16, 2>() : f.template operator()<__nv_bfloat16, 1>();
        default: return V == 2 ? f.template operator()<__half, 2>() : f.template operator()<__half, 1>();
    }
}

// Channels a lane takes: two where every row starts on a multiple of two elements.
int lane_channels(int dtype, size_t D, uintptr_t bits16, uintptr_t bits32) {
    const int es = (int)elem_size(dtype);
    return D % 2 == 0 && common_alignment(bits16, 2 * es) == 2 * es && common_alignment(bits32, 8) == 8 ? 2 : 1;
}

}  // namespace

extern "C" {

int sparbit_scan_plan_create(int n_seqs, const size_t* lengths, size_t channels, int dtype,
                             sparbit_scan_plan_t** out) {
    if (!out) return SPARBIT_ERR_ARG;
    *out = nullptr;
    if (!lengths || n_seqs < 1 || channels < 1 || !known_dtype(dtype)) return SPARBIT_ERR_ARG;
    if (channels > (1u << 20) || n_seqs > 65535) return SPARBIT_ERR_LIMIT;
    const size_t most = ((size_t)1 << 46) / channels;
    size_t rows = 0, pieces = 0;
    for (int s = 0; s < n_seqs; s++) {
        if (lengths[s] > most - rows) return SPARBIT_ERR_OVERFLOW;
        rows += lengths[s];
        pieces += (lengths[s] + kPiece - 1) / kPiece;
        if (pieces > (1u << 24)) return SPARBIT_ERR_LIMIT;
    }
    sparbit_scan_plan_s* p = new (std::nothrow) sparbit_scan_plan_s();
    if (!p) return SPARBIT_ERR_NOMEM;
    try {
        p->n_seqs = n_seqs;
        p->D = (int)channels;
        p->dtype = dtype;
        p->rows = rows;
        p->pieces.reserve(pieces);
        p->seqs.reserve(n_seqs);
        int64_t row = 0;
        for (int s = 0; s < n_seqs; s++) {
            const int32_t first = (int32_t)p->pieces.size();
            for (size_t t = 0; t < lengths[s]; t += kPiece) {
                const size_t left = lengths[s] - t;
                p->pieces.push_back(Piece{row + (int64_t)t, s, (int32_t)(left < kPiece ? left : kPiece)});
            }
            p->seqs.push_back(Seq{first, (int32_t)p->pieces.size() - first});
            row += (int64_t)lengths[s];
        }
    } catch (const std::bad_alloc&) {
        delete p;
        return SPARBIT_ERR_NOMEM;
    }
    *out = p;
    return SPARBIT_OK;
}

int sparbit_scan_plan_destroy(sparbit_scan_plan_t* p) {
    delete p;
    return SPARBIT_OK;
}

size_t sparbit_scan_plan_workspace_bytes(const sparbit_scan_plan_t* p) { return p ? p->work_bytes() : 0; }
size_t sparbit_scan_plan_carry_bytes(const sparbit_scan_plan_t* p) {
    return p ? p->pieces.size() * (size_t)p->D * sizeof(float) : 0;
}

int sparbit_scan_plan_set_workspace(sparbit_scan_plan_t* p, void* dev, size_t bytes) {
    if (!p) return SPARBIT_ERR_ARG;
    if (!dev || bytes < p->work_bytes() || (uintptr_t)dev % 16) return SPARBIT_ERR_WORKSPACE;
    p->work = nullptr;
    CU(cudaGetDevice(&p->device));
    if (!p->pieces.empty())
        CU(cudaMemcpy(dev, p->pieces.data(), p->pieces.size() * sizeof(Piece), cudaMemcpyHostToDevice));
    CU(cudaMemcpy((char*)dev + p->off_seqs(), p->seqs.data(), p->seqs.size() * sizeof(Seq), cudaMemcpyHostToDevice));
    CU(cudaDeviceSynchronize());
    p->work = (char*)dev;
    return SPARBIT_OK;
}

int sparbit_scan_forward(sparbit_scan_plan_t* p, const void* gate, size_t gate_ld, const void* x, size_t x_ld,
                         const float* h0, size_t h0_ld, void* y, size_t y_ld, float* summary, float* carry,
                         void* stream) {
    if (!p) return SPARBIT_ERR_ARG;
    const size_t D = p->D, es = elem_size(p->dtype);
    if (p->rows && (!gate || !x)) return SPARBIT_ERR_ARG;
    if (gate_ld < D || x_ld < D || (y && y_ld < D) || (h0 && h0_ld < D)) return SPARBIT_ERR_ARG;
    const Region rg{gate, p->rows, D * es, gate_ld * es}, rx{x, p->rows, D * es, x_ld * es},
        ry{y, p->rows, D * es, y_ld * es}, rh{h0, (size_t)p->n_seqs, D * 4, h0_ld * 4},
        rs{summary, 1, (size_t)p->n_seqs * 2 * D * 4, 0}, rc{carry, 1, sparbit_scan_plan_carry_bytes(p), 0},
        rw{p->work, 1, p->work_bytes(), 0};
    const Region ins[] = {rg, rx, rh, rw}, outs[] = {ry, rs, rc};
    for (int i = 0; i < 3; i++) {
        for (const Region& in : ins)
            if (regions_overlap(outs[i], in)) return SPARBIT_ERR_ALIAS;
        for (int j = 0; j < i; j++)
            if (regions_overlap(outs[i], outs[j])) return SPARBIT_ERR_ALIAS;
    }
    const int e = ready(p);
    if (e != SPARBIT_OK) return e;
    const uintptr_t bits = (uintptr_t)gate | (uintptr_t)x | (uintptr_t)y | gate_ld * es | x_ld * es | (y ? y_ld * es : 0);
    const int V = lane_channels(p->dtype, D, bits, (uintptr_t)carry);
    return by_type(p->dtype, V, [&]<typename T, int kV>() {
        return run_forward<T, kV>(p, gate, gate_ld, x, x_ld, h0, h0_ld, y, y_ld, summary, carry, (cudaStream_t)stream);
    });
}

int sparbit_scan_backward(sparbit_scan_plan_t* p, const void* gate, size_t gate_ld, const void* x, size_t x_ld,
                          const float* carry, const void* dy, size_t dy_ld, const float* dlast, size_t dlast_ld,
                          void* dgate, size_t dgate_ld, void* dx, size_t dx_ld, float* dsummary, void* stream) {
    if (!p || !dgate != !dx) return SPARBIT_ERR_ARG;
    const size_t D = p->D, es = elem_size(p->dtype);
    if (p->rows && (!gate || !dy || (dx && (!x || !carry)))) return SPARBIT_ERR_ARG;
    if (gate_ld < D || dy_ld < D || (dlast && dlast_ld < D)) return SPARBIT_ERR_ARG;
    if (dx && (x_ld < D || dgate_ld < D || dx_ld < D)) return SPARBIT_ERR_ARG;
    const Region rg{gate, p->rows, D * es, gate_ld * es}, rd{dy, p->rows, D * es, dy_ld * es},
        rx{dx ? x : nullptr, p->rows, D * es, x_ld * es}, rl{dlast, (size_t)p->n_seqs, D * 4, dlast_ld * 4},
        rc{dx ? carry : nullptr, 1, sparbit_scan_plan_carry_bytes(p), 0}, rw{p->work, 1, p->work_bytes(), 0},
        og{dgate, p->rows, D * es, dgate_ld * es}, ox{dx, p->rows, D * es, dx_ld * es},
        os{dsummary, 1, (size_t)p->n_seqs * 2 * D * 4, 0};
    const Region ins[] = {rg, rd, rx, rl, rc, rw}, outs[] = {og, ox, os};
    for (int i = 0; i < 3; i++) {
        for (const Region& in : ins)
            if (regions_overlap(outs[i], in)) return SPARBIT_ERR_ALIAS;
        for (int j = 0; j < i; j++)
            if (regions_overlap(outs[i], outs[j])) return SPARBIT_ERR_ALIAS;
    }
    const int e = ready(p);
    if (e != SPARBIT_OK) return e;
    uintptr_t bits = (uintptr_t)gate | (uintptr_t)dy | gate_ld * es | dy_ld * es;
    if (dx)
        bits |= (uintptr_t)x | (uintptr_t)dgate | (uintptr_t)dx | x_ld * es | dgate_ld * es | dx_ld * es;
    const int V = lane_channels(p->dtype, D, bits, dx ? (uintptr_t)carry : 0);
    return by_type(p->dtype, V, [&]<typename T, int kV>() {
        return run_backward<T, kV>(p, gate, gate_ld, x, x_ld, carry, dy, dy_ld, dlast, dlast_ld, dgate, dgate_ld, dx,
                                   dx_ld, dsummary, (cudaStream_t)stream);
    });
}

int sparbit_scan_step(size_t rows, size_t channels, int dtype, const void* gate, size_t gate_ld, const void* x,
                      size_t x_ld, const int32_t* slots, size_t n_slots, const float* state_in, float* state_out,
                      size_t state_ld, void* y, size_t y_ld, void* stream) {
    if (channels < 1 || !known_dtype(dtype)) return SPARBIT_ERR_ARG;
    if (rows == 0) return SPARBIT_OK;
    if (!gate || !x || !y || (n_slots && (!state_in || !state_out))) return SPARBIT_ERR_ARG;
    if (gate_ld < channels || x_ld < channels || y_ld < channels || state_ld < channels) return SPARBIT_ERR_ARG;
    if (!slots && n_slots < rows) return SPARBIT_ERR_ARG;
    if (channels > (1u << 20) || rows > 0x7fffffffu) return SPARBIT_ERR_LIMIT;
    const size_t es = elem_size(dtype);
    const Region rg{gate, rows, channels * es, gate_ld * es}, rx{x, rows, channels * es, x_ld * es},
        ry{y, rows, channels * es, y_ld * es}, rs{slots, 1, rows * 4, 0},
        ri{state_in, n_slots, channels * 4, state_ld * 4}, ro{state_out, n_slots, channels * 4, state_ld * 4};
    if (regions_overlap(ry, rg) || regions_overlap(ry, rx) || regions_overlap(ry, rs) || regions_overlap(ry, ri) ||
        regions_overlap(ry, ro) || regions_overlap(ro, rg) || regions_overlap(ro, rx) || regions_overlap(ro, rs) ||
        (state_in != state_out && regions_overlap(ro, ri)))
        return SPARBIT_ERR_ALIAS;
    const uintptr_t bits = (uintptr_t)gate | (uintptr_t)x | (uintptr_t)y | gate_ld * es | x_ld * es | y_ld * es;
    const int V = lane_channels(dtype, channels, bits, (uintptr_t)state_in | (uintptr_t)state_out | state_ld * 4);
    return by_type(dtype, V, [&]<typename T, int kV>() {
        CU(launch(scan_step_kernel<T, kV>, dim3((unsigned)rows, (unsigned)((channels + 128 * kV - 1) / (128 * kV))),
                  dim3(128), 0, (cudaStream_t)stream, (const T*)gate, (int64_t)gate_ld, (const T*)x, (int64_t)x_ld,
                  slots, (int64_t)n_slots, (int)channels, state_in, state_out, (int64_t)state_ld, (T*)y,
                  (int64_t)y_ld));
        return (int)SPARBIT_OK;
    });
}

int sparbit_scan_join(int P, int first_rank, int n_ranks, size_t channels, const float* gathered, const float* h0,
                      float* out, size_t out_ld, int reverse, void* stream) {
    if (P < 1 || first_rank < 0 || n_ranks < 1 || n_ranks > P - first_rank || channels < 1) return SPARBIT_ERR_ARG;
    if (!gathered || !out || out_ld < channels) return SPARBIT_ERR_ARG;
    if (channels > (1u << 20) || n_ranks > 65535) return SPARBIT_ERR_LIMIT;
    const Region rg{gathered, 1, (size_t)n_ranks * P * 2 * channels * 4, 0}, rh{h0, 1, channels * 4, 0},
        ro{out, (size_t)n_ranks, channels * 4, out_ld * 4};
    if (regions_overlap(ro, rg) || regions_overlap(ro, rh)) return SPARBIT_ERR_ALIAS;
    CU(launch(scan_join_kernel, dim3((unsigned)((channels + 127) / 128), (unsigned)n_ranks), dim3(128), 0,
              (cudaStream_t)stream, P, first_rank, (int)channels, gathered, h0, out, (int64_t)out_ld, reverse));
    return SPARBIT_OK;
}

}  // extern "C"
