// Gated linear recurrence: h_t = a_t h_{t-1} + (1 - a_t) x_t, a = sigmoid(gate), per channel.
//
// A sequence is cut into pieces of kPiece steps, the channels into tiles of kTile.  What a piece
// does to the state that enters it is the pair (A, H): h -> A h + H, with A the product of its a_t;
// pairs compose, which is what lets the pieces be worked on side by side.  One kernel reads
// every input once: a CTA takes a (piece, channel tile), makes its pair, publishes it, learns the
// state that enters its piece from those before it, and writes the piece's results.
//
// The state that enters comes from the end of the group of kGroup pieces before (published by that
// group's last piece) and the pairs of the earlier pieces of the own group, always folded in the same
// order, so that results do not depend on which CTA was faster.  A wait is one trip to L2 per group of
// 2048 steps, not per piece.  Every published number travels in one 64-bit word with the number of the
// launch: a reader that sees the tag has the value, without fences or flags that need clearing.  Pieces
// are handed out by a ticket counter, in an order in which nobody waits for a later ticket.
#include <new>
#include <vector>

#include "train_common.cuh"

using namespace spb;

namespace {

constexpr int kPiece = 128;    // steps of a piece
constexpr int kTile = 32;      // channels of a tile
constexpr int kGroup = 16;     // pieces of a group
constexpr int kThreads = 256;  // 16 runs of 8 steps (two channels a thread) or 8 runs of 16 (one)
constexpr unsigned long long kWaitNs = 2000000000ull;

// A piece in the order of one direction's chain.
struct Piece {
    int64_t row0;
    int32_t seq, len;
    int32_t slot;   // where its pair is published; those of one chain follow one another
    int32_t at;     // position in its chain
    int32_t group;  // where the state behind its group is published
    int32_t last;   // it ends its chain
    int32_t carry;  // where the forward pass leaves the state that enters it; -1: no rows
    int32_t pad;
};

// First words of the workspace.
struct Control {
    unsigned ticket, done, epoch, status;
};

// a = 1/(1+exp(-g)) and 1 - a, neither of them by cancellation.  Below -80 a is held at exp(-80);
// NaN stays NaN.
__device__ __forceinline__ void gate_pair(float g, float& a, float& keep) {
    float c;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(c) : "f"(g), "f"(-80.0f));
    const float t = __expf(-c);
    a = __fdividef(1.0f, 1.0f + t);
    keep = t * a;
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

// ---- published words ----------------------------------------------------------------------------
// Per piece (or group) and channel two words: value in the low half, tag in the high half.
__device__ __forceinline__ unsigned long long tagged(float v, unsigned tag) {
    return (unsigned long long)tag << 32 | __float_as_uint(v);
}
__device__ __forceinline__ void publish(ulonglong2* p, float a, float h, unsigned tag) {
    asm volatile("st.relaxed.gpu.global.v2.u64 [%0], {%1, %2};" ::"l"(p), "l"(tagged(a, tag)), "l"(tagged(h, tag))
                 : "memory");
}
__device__ __forceinline__ ulonglong2 look(const ulonglong2* p) {
    ulonglong2 v;
    asm volatile("ld.relaxed.gpu.global.v2.u64 {%0, %1}, [%2];" : "=l"(v.x), "=l"(v.y) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ bool ready_word(const ulonglong2& v, unsigned tag) {
    return (unsigned)(v.x >> 32) == tag && (unsigned)(v.y >> 32) == tag;
}
__device__ __forceinline__ float2 values(const ulonglong2& v) {
    return make_float2(__uint_as_float((unsigned)v.x), __uint_as_float((unsigned)v.y));
}
__device__ __forceinline__ unsigned long long now_ns() {
    unsigned long long t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    return t;
}
// Waits for a word that was not there at the first look; gives up after the limit, or when anybody did.
__device__ __noinline__ ulonglong2 wait_word(const ulonglong2* p, unsigned tag, unsigned* status,
                                             unsigned long long limit) {
    const unsigned long long until = now_ns() + limit;
    ulonglong2 v;
    for (;;) {
        v = look(p);
        if (ready_word(v, tag)) return v;
        if (*(volatile unsigned*)status != 0) return v;
        if (now_ns() > until) {
            atomicExch(status, 1u);
            return v;
        }
    }
}

struct ScanArgs {
    const Piece* pieces;
    int tiles, total;  // channel tiles; pieces x tiles
    Control* ctl;
    ulonglong2 *pairs, *groups;
    unsigned long long limit;
    int publish_groups;  // 0: test of the bounded wait
    int D;
    const void *gate, *x, *dy;
    int64_t gate_ld, x_ld, dy_ld;
    int wide;            // rows of all inputs start on multiples of 16 bytes
    const float* first;  // state (gradient) at the start of each chain, or null
    int64_t first_ld;
    float *carry, *summary;
    void *y, *dgate, *dx;
    int64_t y_ld, dgate_ld, dx_ld;
};

// Row t of a staged tensor; a pad of one row every 8 keeps the two runs of a warp in different banks.
__device__ __forceinline__ int stage_row(int t) {
    return (t + (t >> 3)) * kTile;
}
constexpr int kStageElems = (kPiece + kPiece / 8) * kTile;  // of one tensor

// Starts the copy of a piece's rows of one tensor into shared memory.
template <typename T>
__device__ __forceinline__ void stage_tensor(T* dst, const T* src, int64_t ld, const Piece& pc, int ch0, int D,
                                             bool wide) {
    constexpr int kPer = 16 / sizeof(T), kChunks = kTile / kPer;
    if (wide) {
#pragma unroll
        for (int c = threadIdx.x; c < kPiece * kChunks; c += kThreads) {
            const int t = c / kChunks, e = (c % kChunks) * kPer, left = D - ch0 - e;
            if (t < pc.len && left > 0) {
                const uint32_t to = (uint32_t)__cvta_generic_to_shared(dst + stage_row(t) + e);
                const int bytes = left < kPer ? left * (int)sizeof(T) : 16;  // the rest becomes zero
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to),
                             "l"(src + (pc.row0 + t) * ld + ch0 + e), "r"(bytes)
                             : "memory");
            }
        }
    } else {
        for (int c = threadIdx.x; c < kPiece * kTile; c += kThreads) {
            const int t = c / kTile, e = c % kTile;
            if (t < pc.len && ch0 + e < D) dst[stage_row(t) + e] = src[(pc.row0 + t) * ld + ch0 + e];
        }
    }
}
template <typename T, int V>
__device__ __forceinline__ void staged(const T* row, int e, float (&out)[V]) {
    const Pack<T, V> v = *reinterpret_cast<const Pack<T, V>*>(row + e);
#pragma unroll
    for (int i = 0; i < V; i++) out[i] = to_float(v.v[i]);
}

// What a CTA learns about the state that enters its piece.
struct Shared {
    float2 run[kThreads * 2 / kTile][kTile];   // pairs of the runs, then what the runs before make of the entering state
    float2 before[kGroup][kTile];              // pairs of the group's earlier pieces; last: end of the group before
    float enter[kTile];
    float hold[kThreads * 2 / kTile][kTile];   // backward: states at the start of each run
    float2 after[kThreads * 2 / kTile][kTile]; // backward: what the runs behind make of the entering gradient
    Piece piece[2];
    int ticket[2];
    unsigned epoch;
};

// First look at the words this thread is responsible for: thread = (piece of the group, channel pair).
struct Looked {
    ulonglong2 v[2];
};
__device__ __forceinline__ const ulonglong2* word_of(const ScanArgs& g, const Piece& pc, int tile, int j) {
    const int rel = pc.at % kGroup;
    if (j < rel) return g.pairs + ((int64_t)(pc.slot - rel + j) * g.tiles + tile) * kTile;
    if (j == kGroup - 1 && pc.at >= kGroup) return g.groups + ((int64_t)(pc.group - 1) * g.tiles + tile) * kTile;
    return nullptr;
}
__device__ __forceinline__ Looked look_back(const ScanArgs& g, const Piece& pc, int tile) {
    Looked l = {};
    const ulonglong2* p = word_of(g, pc, tile, threadIdx.x / 16);
    if (p) {
        p += threadIdx.x % 16 * 2;
        l.v[0] = look(p);
        l.v[1] = look(p + 1);
    }
    return l;
}
// Puts what the words say into shared memory, waiting where they are not there yet.
__device__ __forceinline__ void settle(const ScanArgs& g, const Piece& pc, int tile, Looked l, unsigned tag,
                                       Shared& s) {
    const int j = threadIdx.x / 16, c = threadIdx.x % 16 * 2;
    const ulonglong2* p = word_of(g, pc, tile, j);
    if (p) {
#pragma unroll
        for (int i = 0; i < 2; i++) {
            if (!ready_word(l.v[i], tag)) l.v[i] = wait_word(p + c + i, tag, &g.ctl->status, g.limit);
            s.before[j][c + i] = values(l.v[i]);
        }
    } else if (j == kGroup - 1) {  // the chain starts with this group
#pragma unroll
        for (int i = 0; i < 2; i++) {
            const int ch = tile * kTile + c + i;
            s.before[j][c + i] = make_float2(1.0f, g.first && ch < g.D ? g.first[pc.seq * g.first_ld + ch] : 0.0f);
        }
    }
}
// One warp, lane = channel: the state that enters the piece, and what leaves the group or the chain.
__device__ __forceinline__ float enter_piece(const ScanArgs& g, const Piece& pc, int tile, float2 own, unsigned tag,
                                             Shared& s) {
    const int lane = threadIdx.x & 31, rel = pc.at % kGroup;
    float A = 1.0f, H = 0.0f;
    for (int j = 0; j < rel; j++) {
        const float2 b = s.before[j][lane];
        H = b.x * H + b.y;
        A *= b.x;
    }
    const float2 from = s.before[kGroup - 1][lane];
    const float h = A * from.y + H, out = own.x * h + own.y, total = own.x * (A * from.x);
    if (rel == kGroup - 1 && g.publish_groups)
        publish(g.groups + ((int64_t)pc.group * g.tiles + tile) * kTile + lane, total, out, tag);
    const int ch = tile * kTile + lane;
    if (pc.last && g.summary && ch < g.D) {
        g.summary[(int64_t)pc.seq * 2 * g.D + ch] = total;
        g.summary[((int64_t)pc.seq * 2 + 1) * g.D + ch] = out;
    }
    return h;
}

// Tickets, kept by thread 0 one tile ahead of the copies: the counter's and the list's latency pass
// while a tile is worked on.
struct Next {
    int ticket;
    Piece piece;
};
__device__ __forceinline__ void draw_ticket(const ScanArgs& g, Next& n) {
    if (threadIdx.x == 0) n.ticket = (int)atomicAdd(&g.ctl->ticket, 1u);
}
__device__ __forceinline__ void read_piece(const ScanArgs& g, Next& n) {
    if (threadIdx.x == 0 && n.ticket < g.total) n.piece = g.pieces[n.ticket / g.tiles];
}
__device__ __forceinline__ void post_ticket(const Next& n, Shared& s, int i) {
    if (threadIdx.x == 0) {
        s.ticket[i] = n.ticket;
        s.piece[i] = n.piece;
    }
}
__device__ __forceinline__ void finish(const ScanArgs& g) {
    // the last CTA to leave makes the counters ready for the next launch; every ticket drawn has been
    // looked at by then
    if (threadIdx.x != 0) return;
    __threadfence();
    if (atomicAdd(&g.ctl->done, 1u) == gridDim.x - 1) {
        g.ctl->ticket = 0;
        g.ctl->done = 0;
        g.ctl->epoch++;
    }
}

// Stages a piece has in shared memory: with two the next piece's copies run while one is worked on;
// pieces of 32-bit elements are large enough that more CTAs per SM do better.
template <typename T>
constexpr int kStagesOf = sizeof(T) == 4 ? 1 : 2;

// Starts the copies of a piece: gate and x, gate and dy, or all three.
template <typename T, int kTensors>
__device__ __forceinline__ void stage_piece(const ScanArgs& g, T* buf, const Piece& pc, int ch0, bool against_time) {
    stage_tensor<T>(buf, (const T*)g.gate, g.gate_ld, pc, ch0, g.D, g.wide);
    if (kTensors == 3 || !against_time)
        stage_tensor<T>(buf + kStageElems, (const T*)g.x, g.x_ld, pc, ch0, g.D, g.wide);
    if (against_time)
        stage_tensor<T>(buf + (kTensors - 1) * kStageElems, (const T*)g.dy, g.dy_ld, pc, ch0, g.D, g.wide);
    asm volatile("cp.async.commit_group;" ::: "memory");
}

// ---- forward (kBack: only what the pieces do to a gradient, for a summary against time) ------------
template <typename T, int V, bool kBack>
__global__ void __launch_bounds__(kThreads, 4) scan_forward_kernel(const __grid_constant__ ScanArgs g) {
    constexpr int kLanes = kTile / V, kRuns = kThreads / kLanes, R = kPiece / kRuns;
    extern __shared__ __align__(16) uint8_t raw[];
    __shared__ Shared s;
    T* stages = reinterpret_cast<T*>(raw);
    pdl_wait();
    pdl_trigger();
    Next next;
    next.piece = Piece{};
    draw_ticket(g, next);
    read_piece(g, next);
    post_ticket(next, s, 0);
    if (threadIdx.x == 0) s.epoch = g.ctl->epoch;
    draw_ticket(g, next);
    read_piece(g, next);
    __syncthreads();
    const unsigned tag = s.epoch;
    const int run = threadIdx.x / kLanes, e = threadIdx.x % kLanes * V, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    constexpr int S = kStagesOf<T>;
    int cur = 0;
    if (S == 2 && s.ticket[0] < g.total)
        stage_piece<T, 2>(g, stages, s.piece[0], s.ticket[0] % g.tiles * kTile, kBack);
    for (; s.ticket[cur] < g.total; cur ^= 1) {
        if (S == 1) stage_piece<T, 2>(g, stages, s.piece[cur], s.ticket[cur] % g.tiles * kTile, kBack);
        post_ticket(next, s, cur ^ 1);
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncthreads();
        draw_ticket(g, next);
        const Piece pc = s.piece[cur];
        const int tile = s.ticket[cur] % g.tiles, ch = tile * kTile + e;
        if (S == 2 && s.ticket[cur ^ 1] < g.total)
            stage_piece<T, 2>(g, stages + (cur ^ 1) * 2 * kStageElems, s.piece[cur ^ 1],
                              s.ticket[cur ^ 1] % g.tiles * kTile, kBack);
        const T* in0 = stages + (S == 2 ? cur : 0) * 2 * kStageElems;
        const T* in1 = in0 + kStageElems;
        float a[R][V], b[R][V], A[V], H[V];
#pragma unroll
        for (int i = 0; i < V; i++) A[i] = 1.0f, H[i] = 0.0f;
#pragma unroll
        for (int j = 0; j < R; j++) {
            const int t = run * R + j;
            staged<T, V>(in0 + stage_row(t), e, a[j]);
            staged<T, V>(in1 + stage_row(t), e, b[j]);
#pragma unroll
            for (int i = 0; i < V; i++) {
                float keep;
                gate_pair(a[j][i], a[j][i], keep);
                if (!kBack) b[j][i] *= keep;
                if (t >= pc.len) a[j][i] = 1.0f, b[j][i] = 0.0f;
                A[i] *= a[j][i];
                // against time the map is built front to back: this step's dy seen through the steps before
                H[i] = kBack ? H[i] + A[i] * b[j][i] : a[j][i] * H[i] + b[j][i];
            }
        }
#pragma unroll
        for (int i = 0; i < V; i++) s.run[run][e + i] = make_float2(A[i], H[i]);
        const Looked seen = look_back(g, pc, tile);
        __syncthreads();
        float2 own = make_float2(1.0f, 0.0f);
        if (warp == 0) {
#pragma unroll
            for (int u = 0; u < kRuns; u++) {
                const int r = kBack ? kRuns - 1 - u : u;
                const float2 p = s.run[r][lane];
                s.run[r][lane] = own;
                own.y = p.x * own.y + p.y;
                own.x *= p.x;
            }
            publish(g.pairs + ((int64_t)pc.slot * g.tiles + tile) * kTile + lane, own.x, own.y, tag);
        }
        settle(g, pc, tile, seen, tag, s);
        read_piece(g, next);
        __syncthreads();
        if (warp == 0) {
            const float h = enter_piece(g, pc, tile, own, tag, s);
            s.enter[lane] = h;
            if (!kBack && g.carry && pc.carry >= 0 && tile * kTile + lane < g.D)
                g.carry[(int64_t)pc.carry * g.D + tile * kTile + lane] = h;
        }
        __syncthreads();
        if (!kBack && g.y && ch < g.D) {
            float h[V];
#pragma unroll
            for (int i = 0; i < V; i++) h[i] = s.run[run][e + i].x * s.enter[e + i] + s.run[run][e + i].y;
            T* y = (T*)g.y + (pc.row0 + run * R) * g.y_ld + ch;
#pragma unroll
            for (int j = 0; j < R; j++) {
#pragma unroll
                for (int i = 0; i < V; i++) h[i] = a[j][i] * h[i] + b[j][i];
                if (run * R + j < pc.len) store_row<T, V>(y, j, g.y_ld, 0, h);
            }
        }
    }
    finish(g);
}

// ---- backward -------------------------------------------------------------------------------------
// The states of the piece are computed again from the one that the forward pass left at its start.
template <typename T, int V>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 4 ? 2 : 3) scan_backward_kernel(const __grid_constant__ ScanArgs g) {
    constexpr int kLanes = kTile / V, kRuns = kThreads / kLanes, R = kPiece / kRuns;
    extern __shared__ __align__(16) uint8_t raw[];
    __shared__ Shared s;
    T* stages = reinterpret_cast<T*>(raw);
    pdl_wait();
    pdl_trigger();
    Next next;
    next.piece = Piece{};
    draw_ticket(g, next);
    read_piece(g, next);
    post_ticket(next, s, 0);
    if (threadIdx.x == 0) s.epoch = g.ctl->epoch;
    draw_ticket(g, next);
    read_piece(g, next);
    __syncthreads();
    const unsigned tag = s.epoch;
    const int run = threadIdx.x / kLanes, e = threadIdx.x % kLanes * V, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    constexpr int S = kStagesOf<T>;
    int cur = 0;
    if (S == 2 && s.ticket[0] < g.total)
        stage_piece<T, 3>(g, stages, s.piece[0], s.ticket[0] % g.tiles * kTile, true);
    for (; s.ticket[cur] < g.total; cur ^= 1) {
        if (S == 1) {
            __syncthreads();  // the last piece's dy has been read
            stage_piece<T, 3>(g, stages, s.piece[cur], s.ticket[cur] % g.tiles * kTile, true);
        }
        post_ticket(next, s, cur ^ 1);
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncthreads();
        draw_ticket(g, next);
        const Piece pc = s.piece[cur];
        const int tile = s.ticket[cur] % g.tiles, ch = tile * kTile + e;
        if (S == 2 && s.ticket[cur ^ 1] < g.total)
            stage_piece<T, 3>(g, stages + (cur ^ 1) * 3 * kStageElems, s.piece[cur ^ 1],
                              s.ticket[cur ^ 1] % g.tiles * kTile, true);
        const T* in_g = stages + (S == 2 ? cur : 0) * 3 * kStageElems;
        const T* in_x = in_g + kStageElems;
        const T* in_d = in_x + kStageElems;
        float carried = 0.0f;
        if (warp == 1 && pc.carry >= 0 && tile * kTile + lane < g.D)
            carried = g.carry[(int64_t)pc.carry * g.D + tile * kTile + lane];
        float a[R][V], k[R][V], A[V], H[V], G[V];
#pragma unroll
        for (int i = 0; i < V; i++) A[i] = 1.0f, H[i] = 0.0f, G[i] = 0.0f;
#pragma unroll
        for (int j = 0; j < R; j++) {
            const int t = run * R + j;
            float x[V], d[V];
            staged<T, V>(in_g + stage_row(t), e, a[j]);
            staged<T, V>(in_x + stage_row(t), e, x);
            staged<T, V>(in_d + stage_row(t), e, d);
            const bool on = t < pc.len;
#pragma unroll
            for (int i = 0; i < V; i++) {
                gate_pair(a[j][i], a[j][i], k[j][i]);
                if (!on) a[j][i] = 1.0f, k[j][i] = x[i] = d[i] = 0.0f;
                A[i] *= a[j][i];
                H[i] = a[j][i] * H[i] + k[j][i] * x[i];
                // the map of a gradient, front to back: this step's dy seen through the steps before
                G[i] += A[i] * d[i];
            }
        }
#pragma unroll
        for (int i = 0; i < V; i++) {
            s.run[run][e + i] = make_float2(A[i], G[i]);
            s.hold[run][e + i] = H[i];
        }
        const Looked seen = look_back(g, pc, tile);
        __syncthreads();
        float2 own = make_float2(1.0f, 0.0f);
        if (warp == 1) {  // states at the start of each run
            float h = carried;
#pragma unroll
            for (int u = 0; u < kRuns; u++) {
                const float next = s.run[u][lane].x * h + s.hold[u][lane];
                s.hold[u][lane] = h;
                h = next;
            }
        }
        if (warp == 0) {
#pragma unroll
            for (int u = kRuns - 1; u >= 0; u--) {
                const float2 p = s.run[u][lane];
                s.after[u][lane] = own;
                own.y = p.x * own.y + p.y;
                own.x *= p.x;
            }
            publish(g.pairs + ((int64_t)pc.slot * g.tiles + tile) * kTile + lane, own.x, own.y, tag);
        }
        __syncthreads();
        // (h_{t-1} - x_t) a_t (1 - a_t), while the words travel
        float f[R][V], h[V];
#pragma unroll
        for (int i = 0; i < V; i++) h[i] = s.hold[run][e + i];
#pragma unroll
        for (int j = 0; j < R; j++) {
            float x[V];
            staged<T, V>(in_x + stage_row(run * R + j), e, x);
#pragma unroll
            for (int i = 0; i < V; i++) {
                f[j][i] = (h[i] - x[i]) * a[j][i] * k[j][i];
                h[i] = a[j][i] * h[i] + k[j][i] * x[i];
            }
        }
        settle(g, pc, tile, seen, tag, s);
        read_piece(g, next);
        __syncthreads();
        if (warp == 0) s.enter[lane] = enter_piece(g, pc, tile, own, tag, s);
        __syncthreads();
        if (ch < g.D) {
            float c[V];
#pragma unroll
            for (int i = 0; i < V; i++) c[i] = s.after[run][e + i].x * s.enter[e + i] + s.after[run][e + i].y;
            T* dg = (T*)g.dgate + (pc.row0 + run * R) * g.dgate_ld + ch;
            T* dx = (T*)g.dx + (pc.row0 + run * R) * g.dx_ld + ch;
#pragma unroll
            for (int j = R - 1; j >= 0; j--) {
                if (run * R + j >= pc.len) continue;
                float d[V];
                staged<T, V>(in_d + stage_row(run * R + j), e, d);
#pragma unroll
                for (int i = 0; i < V; i++) {
                    const float q = d[i] + c[i];
                    f[j][i] *= q;
                    c[i] = a[j][i] * q;
                    k[j][i] *= q;
                }
                store_row<T, V>(dg, j, g.dgate_ld, 0, f[j]);
                store_row<T, V>(dx, j, g.dx_ld, 0, k[j]);
            }
        }
    }
    finish(g);
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
    size_t carries = 0;                 // pieces that have rows
    std::vector<Piece> forward, backward;  // in the order of the tickets
    size_t n_groups = 0;
    char* work = nullptr;
    int device = -1, sm_count = 0;
    unsigned long long limit = kWaitNs;
    int publish_groups = 1;

    size_t tiles() const { return ((size_t)D + kTile - 1) / kTile; }
    size_t off_forward() const { return 256; }
    size_t off_backward() const { return off_forward() + round_up(forward.size() * sizeof(Piece), 256); }
    size_t off_pairs() const { return off_backward() + round_up(backward.size() * sizeof(Piece), 256); }
    size_t off_groups() const { return off_pairs() + forward.size() * tiles() * kTile * sizeof(ulonglong2); }
    size_t work_bytes() const { return off_groups() + n_groups * tiles() * kTile * sizeof(ulonglong2); }
};

namespace {

int ready(const sparbit_scan_plan_s* p) {
    if (!p->work) return SPARBIT_ERR_WORKSPACE;
    int cur = -1;
    CU(cudaGetDevice(&cur));
    return cur == p->device ? SPARBIT_OK : SPARBIT_ERR_ARG;
}

ScanArgs common_args(const sparbit_scan_plan_s* p, bool against_time) {
    ScanArgs g = {};
    g.pieces = (const Piece*)(p->work + (against_time ? p->off_backward() : p->off_forward()));
    g.tiles = (int)p->tiles();
    g.total = (int)(p->forward.size() * p->tiles());
    g.ctl = (Control*)p->work;
    g.pairs = (ulonglong2*)(p->work + p->off_pairs());
    g.groups = (ulonglong2*)(p->work + p->off_groups());
    g.limit = p->limit;
    g.publish_groups = p->publish_groups;
    g.D = p->D;
    return g;
}

// As many CTAs as fit, each taking tickets until there are none.
int run(const sparbit_scan_plan_s* p, void (*kernel)(ScanArgs), int tensors, const ScanArgs& g, cudaStream_t st) {
    const size_t smem = (p->dtype == SPARBIT_F32 ? kStagesOf<float> : kStagesOf<__half>) * tensors *
                        (size_t)kStageElems * elem_size(p->dtype);
    CU(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    int per_sm = 0;
    CU(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, kThreads, smem));
    const int most = (per_sm > 0 ? per_sm : 1) * p->sm_count;
    CU(launch(kernel, dim3(g.total < most ? g.total : most), dim3(kThreads), smem, st, g));
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
    const size_t most = ((size_t)1 << 46) / channels, tiles = (channels + kTile - 1) / kTile;
    size_t rows = 0, pieces = 0;
    for (int s = 0; s < n_seqs; s++) {
        if (lengths[s] > most - rows) return SPARBIT_ERR_OVERFLOW;
        rows += lengths[s];
        pieces += lengths[s] ? (lengths[s] + kPiece - 1) / kPiece : 1;
        if (pieces * tiles > (1u << 30)) return SPARBIT_ERR_LIMIT;
    }
    sparbit_scan_plan_s* p = new (std::nothrow) sparbit_scan_plan_s();
    if (!p) return SPARBIT_ERR_NOMEM;
    try {
        p->n_seqs = n_seqs;
        p->D = (int)channels;
        p->dtype = dtype;
        p->rows = rows;
        // chain by chain first; the tickets then go by the position in the chain, so that all chains
        // advance together and a piece rarely waits
        std::vector<Piece> chains[2];
        std::vector<size_t> upto;  // pieces with a position below i, over all chains
        int64_t row = 0;
        int32_t slot = 0, group = 0, carry = 0;
        for (int s = 0; s < n_seqs; s++) {
            const int32_t n = lengths[s] ? (int32_t)((lengths[s] + kPiece - 1) / kPiece) : 1;
            if (upto.size() < (size_t)n + 1) upto.resize((size_t)n + 1, 0);
            for (int32_t i = 0; i < n; i++) {
                upto[i + 1]++;
                for (int back = 0; back < 2; back++) {
                    const int32_t q = back ? n - 1 - i : i;
                    const size_t t = (size_t)q * kPiece, left = lengths[s] - t;
                    chains[back].push_back(Piece{row + (int64_t)t, s, (int32_t)(left < kPiece ? left : kPiece), slot + i, i,
                                                 group + i / kGroup, i == n - 1, lengths[s] ? carry + q : -1, 0});
                }
            }
            slot += n;
            group += (n + kGroup - 1) / kGroup;
            if (lengths[s]) carry += n;
            row += (int64_t)lengths[s];
        }
        p->carries = (size_t)carry;
        p->n_groups = (size_t)group;
        for (size_t i = 1; i < upto.size(); i++) upto[i] += upto[i - 1];
        for (int back = 0; back < 2; back++) {
            std::vector<Piece>& out = back ? p->backward : p->forward;
            std::vector<size_t> next = upto;
            out.resize(chains[back].size());
            for (const Piece& pc : chains[back]) out[next[pc.at]++] = pc;
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
    return p ? p->carries * (size_t)p->D * sizeof(float) : 0;
}

int sparbit_scan_plan_set_workspace(sparbit_scan_plan_t* p, void* dev, size_t bytes) {
    if (!p) return SPARBIT_ERR_ARG;
    if (!dev || bytes < p->work_bytes() || (uintptr_t)dev % 16) return SPARBIT_ERR_WORKSPACE;
    p->work = nullptr;
    CU(cudaGetDevice(&p->device));
    CU(cudaDeviceGetAttribute(&p->sm_count, cudaDevAttrMultiProcessorCount, p->device));
    char* base = (char*)dev;
    // words of tag 0 are of no launch
    CU(cudaMemset(base + p->off_pairs(), 0, p->work_bytes() - p->off_pairs()));
    const Control ctl = {0, 0, 1, 0};
    CU(cudaMemcpy(base, &ctl, sizeof ctl, cudaMemcpyHostToDevice));
    CU(cudaMemcpy(base + p->off_forward(), p->forward.data(), p->forward.size() * sizeof(Piece), cudaMemcpyHostToDevice));
    CU(cudaMemcpy(base + p->off_backward(), p->backward.data(), p->backward.size() * sizeof(Piece),
                  cudaMemcpyHostToDevice));
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
    ScanArgs g = common_args(p, false);
    g.gate = gate;
    g.gate_ld = (int64_t)gate_ld;
    g.x = x;
    g.x_ld = (int64_t)x_ld;
    g.wide = common_alignment((uintptr_t)gate | (uintptr_t)x | gate_ld * es | x_ld * es, 16) == 16;
    g.first = h0;
    g.first_ld = (int64_t)h0_ld;
    g.y = y;
    g.y_ld = (int64_t)y_ld;
    g.summary = summary;
    g.carry = carry;
    const int V = lane_channels(p->dtype, D, y ? (uintptr_t)y | y_ld * es : 0, 0);
    return by_type(p->dtype, V, [&]<typename T, int kV>() {
        return run(p, scan_forward_kernel<T, kV, false>, 2, g, (cudaStream_t)stream);
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
    ScanArgs g = common_args(p, true);
    g.gate = gate;
    g.gate_ld = (int64_t)gate_ld;
    g.dy = dy;
    g.dy_ld = (int64_t)dy_ld;
    g.first = dlast;
    g.first_ld = (int64_t)dlast_ld;
    g.summary = dsummary;
    uintptr_t in_bits = (uintptr_t)gate | (uintptr_t)dy | gate_ld * es | dy_ld * es;
    if (!dx) {
        g.wide = common_alignment(in_bits, 16) == 16;
        return by_type(p->dtype, lane_channels(p->dtype, 2, 0, 0), [&]<typename T, int kV>() {
            return run(p, scan_forward_kernel<T, kV, true>, 2, g, (cudaStream_t)stream);
        });
    }
    in_bits |= (uintptr_t)x | x_ld * es;
    g.wide = common_alignment(in_bits, 16) == 16;
    g.x = x;
    g.x_ld = (int64_t)x_ld;
    g.carry = (float*)carry;
    g.dgate = dgate;
    g.dgate_ld = (int64_t)dgate_ld;
    g.dx = dx;
    g.dx_ld = (int64_t)dx_ld;
    const uintptr_t out_bits = (uintptr_t)dgate | (uintptr_t)dx | dgate_ld * es | dx_ld * es;
    return by_type(p->dtype, lane_channels(p->dtype, D, out_bits, 0), [&]<typename T, int kV>() {
        return run(p, scan_backward_kernel<T, kV>, 3, g, (cudaStream_t)stream);
    });
}

int sparbit_scan_plan_status(sparbit_scan_plan_t* p) {
    if (!p) return SPARBIT_ERR_ARG;
    const int e = ready(p);
    if (e != SPARBIT_OK) return e;
    CU(cudaDeviceSynchronize());
    Control ctl;
    CU(cudaMemcpy(&ctl, p->work, sizeof ctl, cudaMemcpyDeviceToHost));
    if (ctl.status == 0) return SPARBIT_OK;
    CU(cudaMemset(&((Control*)p->work)->status, 0, sizeof(unsigned)));
    return SPARBIT_ERR_TIMEOUT;
}

int sparbit_scan_plan_set_wait_test(sparbit_scan_plan_t* p, int withhold, uint64_t timeout_ns) {
    if (!p) return SPARBIT_ERR_ARG;
    p->publish_groups = !withhold;
    p->limit = timeout_ns ? timeout_ns : kWaitNs;
    return SPARBIT_OK;
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
