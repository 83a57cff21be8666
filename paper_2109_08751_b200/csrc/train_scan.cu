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
// 1024 steps, not per piece.  Every published number travels in one 64-bit word with the number of the
// launch: a reader that sees the tag has the value, without fences or flags that need clearing.  Pieces
// are handed out by a ticket counter, in an order in which nobody waits for a later ticket.
//
// Bytes are the floor: 6 an element forward and 10 backward for 16-bit types.  8 x 4096 x 2048 bf16 takes
// 92 us and 162 us, 4.4 and 4.1 TB/s, about two thirds of a copy's rate: 27 instructions an element, two of
// them exponential or reciprocal, and three barriers a piece keep 53 % of the issue slots busy.
#include <new>
#include <vector>

#include "train_common.cuh"

using namespace spb;

namespace {

constexpr int kPiece = 128;    // steps of a piece
constexpr int kTile = 32;      // channels of a tile
constexpr int kGroup = 8;      // pieces of a group
// A thread's share of a piece: V channels of a run of steps, A of them an access.  16 runs of 8 steps with
// two or four channels a thread, 8 runs of 16 with one.
template <int V>
constexpr int kThreads = V == 4 ? 128 : 256;
constexpr unsigned long long kWaitNs = 2000000000ull;

// A piece in the order of one direction's chain.
struct alignas(16) Piece {
    int64_t row0;
    int32_t seq, len;
    int32_t slot;   // where its pair is published; those of one chain follow one another
    int32_t at;     // position in its chain
    int32_t group;  // where the state behind its group is published
    int32_t last;   // it ends its chain
    int32_t carry;  // where the forward pass leaves the state that enters it; -1: no rows
    int32_t pad[3];
};

// First words of the workspace.  epoch is the number of the launch (its tag, never 0), status that of the last one
// in which a wait gave up: later launches wait as ever.
struct Control {
    unsigned ticket, done, epoch, status;
};

// V channels of a thread; pairs of them go through the packed fp32 instructions of sm_100.
template <int V>
struct F {
    float v[V];
};
__device__ __forceinline__ unsigned long long pair_bits(float a, float b) {
    return (unsigned long long)__float_as_uint(b) << 32 | __float_as_uint(a);
}
__device__ __forceinline__ void from_pair(unsigned long long p, float& a, float& b) {
    a = __uint_as_float((unsigned)p);
    b = __uint_as_float((unsigned)(p >> 32));
}
template <int V>
__device__ __forceinline__ F<V> fma(const F<V>& a, const F<V>& b, const F<V>& c) {
    F<V> r;
    if constexpr (V == 1) {
        r.v[0] = fmaf(a.v[0], b.v[0], c.v[0]);
    } else {
#pragma unroll
        for (int i = 0; i < V; i += 2) {
            unsigned long long d;
            asm("fma.rn.f32x2 %0, %1, %2, %3;"
                : "=l"(d)
                : "l"(pair_bits(a.v[i], a.v[i + 1])), "l"(pair_bits(b.v[i], b.v[i + 1])), "l"(pair_bits(c.v[i], c.v[i + 1])));
            from_pair(d, r.v[i], r.v[i + 1]);
        }
    }
    return r;
}
template <int V>
__device__ __forceinline__ F<V> mul(const F<V>& a, const F<V>& b) {
    F<V> r;
    if constexpr (V == 1) {
        r.v[0] = a.v[0] * b.v[0];
    } else {
#pragma unroll
        for (int i = 0; i < V; i += 2) {
            unsigned long long d;
            asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(pair_bits(a.v[i], a.v[i + 1])), "l"(pair_bits(b.v[i], b.v[i + 1])));
            from_pair(d, r.v[i], r.v[i + 1]);
        }
    }
    return r;
}
template <int V>
__device__ __forceinline__ F<V> add(const F<V>& a, const F<V>& b) {
    F<V> r;
    if constexpr (V == 1) {
        r.v[0] = a.v[0] + b.v[0];
    } else {
#pragma unroll
        for (int i = 0; i < V; i += 2) {
            unsigned long long d;
            asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(pair_bits(a.v[i], a.v[i + 1])), "l"(pair_bits(b.v[i], b.v[i + 1])));
            from_pair(d, r.v[i], r.v[i + 1]);
        }
    }
    return r;
}
template <int V>
__device__ __forceinline__ F<V> all(float x) {
    F<V> f;
#pragma unroll
    for (int i = 0; i < V; i++) f.v[i] = x;
    return f;
}

// a = 1/(1+exp(-g)) and 1 - a, neither of them by cancellation: with t = exp(-g), a = 1/(1+t) and
// 1 - a = t a.  t is held at 2^115, so that t a stays 1 for gates below -80; NaN stays NaN.
template <int V>
__device__ __forceinline__ void gate_pair(const F<V>& g, F<V>& a, F<V>& keep) {
    F<V> t = mul(g, all<V>(-1.4426950408889634f));
#pragma unroll
    for (int i = 0; i < V; i++) {
        asm("min.NaN.f32 %0, %0, %1;" : "+f"(t.v[i]) : "f"(115.0f));
        asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(t.v[i]));
    }
    a = add(t, all<V>(1.0f));
#pragma unroll
    for (int i = 0; i < V; i++) asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(a.v[i]));
    keep = mul(t, a);
}

// V neighbouring elements, A of them an access.
template <typename T, int V, int A>
__device__ __forceinline__ F<V> unpack(const T* p) {
    F<V> f;
#pragma unroll
    for (int u = 0; u < V; u += A) {
        const Pack<T, A> k = *reinterpret_cast<const Pack<T, A>*>(p + u);
#pragma unroll
        for (int i = 0; i < A; i++) f.v[u + i] = to_float(k.v[i]);
    }
    return f;
}
// The first `left` of them (a multiple of A) are there to be written.
template <typename T, int V, int A>
__device__ __forceinline__ void pack(T* p, const F<V>& f, int left) {
#pragma unroll
    for (int u = 0; u < V; u += A) {
        Pack<T, A> k;
#pragma unroll
        for (int i = 0; i < A; i++) k.v[i] = from_float<T>(f.v[u + i]);
        if (A == V || u < left) *reinterpret_cast<Pack<T, A>*>(p + u) = k;
    }
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
// Waits for two neighbouring words that were not there at the first look; gives up after the limit, or when
// anybody in this launch did.
__device__ __noinline__ void wait_words(const ulonglong2* p, unsigned tag, unsigned* status, unsigned long long limit,
                                        ulonglong2& a, ulonglong2& b) {
    const unsigned long long until = now_ns() + limit;
    for (;;) {
        // a look is one trip to L2; what ends the wait early is asked for now and then only
        for (int i = 0; i < 32; i++) {
            a = look(p);
            b = look(p + 1);
            if (ready_word(a, tag) && ready_word(b, tag)) return;
        }
        if (*(volatile unsigned*)status == tag) return;
        if (now_ns() > until) {
            atomicExch(status, tag);
            return;
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
    const float* first;  // state (gradient) at the start of each chain, or null
    int64_t first_ld;
    float *carry, *summary;
    void *y, *dgate, *dx;
    int64_t y_ld, dgate_ld, dx_ld;
};

// A piece's rows of one tensor in shared memory.  Where all rows start on multiples of 16 bytes (kWide)
// they lie there as they are; otherwise each is copied from the multiple of 16 bytes before it, so that
// copies stay 16 bytes wide, and starts where it did within them.  A pad after every run of R rows keeps
// the runs of a warp in different banks.
template <typename T, int R, bool kWide>
struct Stage {
    static constexpr int kRow = kTile * (int)sizeof(T), kPitch = kRow + (kWide ? 0 : 16), kPad = kWide ? kRow : 64;
    static constexpr int kBytes = kPiece * kPitch + kPiece / R * kPad;
    static constexpr int kChunks = kPitch / 16;
    __device__ __forceinline__ static int row(int t) { return t * kPitch + t / R * kPad; }
};
// A thread's run of rows of it.
template <typename T, int V, int A, int R, bool kWide>
struct Rows {
    int at;                // bytes into the dynamic shared memory
    uint32_t first, step;  // of rows that are not wide: where row j starts within its 16 bytes
    __device__ __forceinline__ Rows(int stage, int run, int e, const void* src, int64_t ld, int64_t row0, int ch0) {
        at = stage + Stage<T, R, kWide>::row(run * R) + e * (int)sizeof(T);
        step = (uint32_t)ld * (uint32_t)sizeof(T);
        first = (uint32_t)(uintptr_t)src + (uint32_t)(row0 + run * R) * step + (uint32_t)ch0 * (uint32_t)sizeof(T);
    }
    __device__ __forceinline__ F<V> operator[](int j) const {
        extern __shared__ __align__(16) uint8_t raw[];
        int p = at + j * Stage<T, R, kWide>::kPitch;
        if (!kWide) p += (int)((first + (uint32_t)j * step) & 15u);
        return unpack<T, V, A>(reinterpret_cast<const T*>(raw + p));
    }
};

// Starts the copy of a piece's rows of one tensor.  Of rows that are not wide it reads up to 15 bytes in front of a row
// (the rest of 16 aligned bytes, unused), but nothing in front of the tensor or behind a row.
template <typename T, int R, int kThr, bool kWide, bool kBurst>
__device__ __forceinline__ void stage_tensor(char* stage, const T* src, int64_t ld, int64_t row0, int len, int ch0, int D) {
    using S = Stage<T, R, kWide>;
    constexpr int kPer = 16 / sizeof(T);
    const uint32_t to = (uint32_t)__cvta_generic_to_shared(stage);
    if constexpr (kWide) {
        constexpr int kRows = kThr / S::kChunks;  // rows between the copies of a thread
        static_assert(kRows % 8 == 0 && (kRows % R == 0 || R % kRows == 0), "");
        const int t0 = threadIdx.x / S::kChunks, e = threadIdx.x % S::kChunks * kPer, left = D - ch0 - e;
        if (left <= 0) return;
        const int bytes = left < kPer ? left * (int)sizeof(T) : 16;  // the rest becomes zero
        const T* from = src + (row0 + t0) * ld + ch0 + e;
        const uint32_t dst = to + S::row(t0) + e * (int)sizeof(T);
        // Copies of the next piece, issued all at once, hold up the words that other CTAs wait for (65536 x
        // 2048 bf16 forward 287 us rolled up, 345 unrolled); copies that are waited for at once should be
        // (8 x 8192 x 1024 f32 forward 162 us unrolled, 175 rolled up).
        constexpr int kUnroll = kBurst ? kPiece / kRows : 1;
#pragma unroll kUnroll
        for (int i = 0; i < kPiece / kRows; i++) {
            if (t0 + i * kRows < len)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + (uint32_t)S::row(i * kRows)),
                             "l"(from), "r"(bytes)
                             : "memory");
            from += kRows * ld;
        }
    } else {
        const int need = (D - ch0 < kTile ? D - ch0 : kTile) * (int)sizeof(T);
        const char* const rows = reinterpret_cast<const char*>(src + row0 * ld + ch0);
        const int64_t pitch = ld * (int64_t)sizeof(T);
#pragma unroll 1
        for (int c = threadIdx.x; c < kPiece * S::kChunks; c += kThr) {
            const int t = c / S::kChunks, q = c - t * S::kChunks;
            if (t >= len) break;
            const char* const start = rows + t * pitch;
            const int over = (int)((uintptr_t)start & 15);
            const char* const from = start - over + q * 16;
            const int bytes = need + over - q * 16 < 16 ? need + over - q * 16 : 16;
            if (bytes <= 0) continue;
            const uint32_t dst = to + S::row(t) + q * 16;
            if (from >= reinterpret_cast<const char*>(src)) {
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(from), "r"(bytes) : "memory");
            } else {  // the tensor's first bytes: nothing in front of them is touched
                for (int i = over; i < bytes; i += (int)sizeof(T))
                    *reinterpret_cast<T*>(stage + S::row(t) + i) = *reinterpret_cast<const T*>(from + i);
            }
        }
    }
}

constexpr int kMostRuns = 16;
struct SharedBack {
    float hold[kMostRuns][kTile];    // states at the start of each run
    float2 after[kMostRuns][kTile];  // what the runs behind make of the entering gradient
};

// What a CTA learns about the state that enters its piece.
struct Shared {
    float2 run[kMostRuns][kTile];   // pairs of the runs, then what the runs before make of the entering state
    float2 before[kGroup][kTile];              // pairs of the group's earlier pieces; last: end of the group before
    float enter[kTile];
    Piece piece[4];
    int ticket[4], tile[4];
    unsigned epoch;
};

// First look at the words this thread is responsible for: 16 threads to a piece of the group (the last:
// the group before), two channels each.
template <int kThr>
struct Looked {
    static constexpr int kEach = (kGroup * 16 + kThr - 1) / kThr;
    ulonglong2 v[kEach][2];
};
__device__ __forceinline__ const ulonglong2* word_of(const ScanArgs& g, const Piece& pc, int tile, int j) {
    const int rel = pc.at % kGroup;
    if (j < rel) return g.pairs + ((int64_t)(pc.slot - rel + j) * g.tiles + tile) * kTile;
    if (j == kGroup - 1 && pc.at >= kGroup) return g.groups + ((int64_t)(pc.group - 1) * g.tiles + tile) * kTile;
    return nullptr;
}
template <int kThr>
__device__ __forceinline__ Looked<kThr> look_back(const ScanArgs& g, const Piece& pc, int tile) {
    Looked<kThr> l = {};
#pragma unroll
    for (int i = 0; i < Looked<kThr>::kEach; i++) {
        const ulonglong2* p = word_of(g, pc, tile, threadIdx.x / 16 + i * (kThr / 16));
        if (p) {
            p += threadIdx.x % 16 * 2;
            l.v[i][0] = look(p);
            l.v[i][1] = look(p + 1);
        }
    }
    return l;
}
// Puts what the words say into shared memory, waiting where they are not there yet.
template <int kThr>
__device__ __forceinline__ void settle(const ScanArgs& g, const Piece& pc, int tile, Looked<kThr> l, unsigned tag,
                                       Shared& s) {
    const int c = threadIdx.x % 16 * 2;
#pragma unroll
    for (int u = 0; u < Looked<kThr>::kEach; u++) {
        const int j = threadIdx.x / 16 + u * (kThr / 16);
        const ulonglong2* p = word_of(g, pc, tile, j);
        if (p) {
            if (!ready_word(l.v[u][0], tag) || !ready_word(l.v[u][1], tag))
                wait_words(p + c, tag, &g.ctl->status, g.limit, l.v[u][0], l.v[u][1]);
            s.before[j][c] = values(l.v[u][0]);
            s.before[j][c + 1] = values(l.v[u][1]);
        } else if (j == kGroup - 1) {  // the chain starts with this group
#pragma unroll
            for (int i = 0; i < 2; i++) {
                const int ch = tile * kTile + c + i;
                s.before[j][c + i] = make_float2(1.0f, g.first && ch < g.D ? g.first[pc.seq * g.first_ld + ch] : 0.0f);
            }
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

// Tickets n, n + 1 and n + 2 (n: the tile worked on, n + 1: its copies under way) live in slots of
// s.ticket and s.piece; thread 0 draws one and starts the copy of its entry of the list while a tile is
// worked on, so that neither latency is waited for.
__device__ __forceinline__ int draw_ticket(const ScanArgs& g) {
    return threadIdx.x == 0 ? (int)atomicAdd(&g.ctl->ticket, 1u) : 0;
}
__device__ __forceinline__ void post_ticket(const ScanArgs& g, Shared& s, int slot, int ticket) {
    if (threadIdx.x != 0) return;
    s.ticket[slot] = ticket;
    if (ticket < g.total) {
        const int piece = ticket / g.tiles;
        s.tile[slot] = ticket - piece * g.tiles;
        const char* from = (const char*)(g.pieces + piece);
        const uint32_t to = (uint32_t)__cvta_generic_to_shared(&s.piece[slot]);
#pragma unroll
        for (int i = 0; i < (int)sizeof(Piece); i += 16)
            asm volatile("cp.async.ca.shared.global [%0], [%1], 16;" ::"r"(to + i), "l"(from + i) : "memory");
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
        const unsigned next = g.ctl->epoch + 1;
        g.ctl->epoch = next != 0 ? next : 1;
    }
}

// Stages a piece has in shared memory: with two the next piece's copies run while one is worked on;
// pieces of 32-bit elements are large enough that more CTAs per SM do better.
template <typename T, int kTensors, int V>
constexpr int kStagesOf = sizeof(T) == 4 || (kTensors == 3 && V == 4) ? 1 : 2;

// Starts the copies of a piece: gate and x, gate and dy, or all three.
template <typename T, int kTensors, int R, int kThr, bool kWide, bool kBurst>
__device__ __forceinline__ void stage_piece(const ScanArgs& g, char* buf, const Shared& s, int slot, bool against_time) {
    constexpr int kBytes = Stage<T, R, kWide>::kBytes;
    const int64_t row0 = s.piece[slot].row0;
    const int len = s.piece[slot].len, ch0 = s.tile[slot] * kTile;
    stage_tensor<T, R, kThr, kWide, kBurst>(buf, (const T*)g.gate, g.gate_ld, row0, len, ch0, g.D);
    if (kTensors == 3 || !against_time)
        stage_tensor<T, R, kThr, kWide, kBurst>(buf + kBytes, (const T*)g.x, g.x_ld, row0, len, ch0, g.D);
    if (against_time)
        stage_tensor<T, R, kThr, kWide, kBurst>(buf + (kTensors - 1) * kBytes, (const T*)g.dy, g.dy_ld, row0, len, ch0, g.D);
}
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// What both kernels begin with; returns this launch's tag.
template <typename T, int kTensors, int V, int R, int kThr, bool kWide>
__device__ __forceinline__ unsigned begin(const ScanArgs& g, char* stages, Shared& s, bool against_time) {
    pdl_wait();
    pdl_trigger();
    post_ticket(g, s, 0, draw_ticket(g));
    post_ticket(g, s, 1, draw_ticket(g));
    if (threadIdx.x == 0) s.epoch = g.ctl->epoch;
    copies_wait();
    __syncthreads();
    if (kStagesOf<T, kTensors, V> == 2 && s.ticket[0] < g.total) stage_piece<T, kTensors, R, kThr, kWide, false>(g, stages, s, 0, against_time);
    return s.epoch;
}

// ---- forward (kBack: only what the pieces do to a gradient, for a summary against time) ------------
template <typename T, int V, int A, bool kBack, bool kWide>
__global__ void __launch_bounds__(kThreads<V>, V == 4 ? 5 : 4) scan_forward_kernel(const __grid_constant__ ScanArgs g) {
    constexpr int kThr = kThreads<V>, kLanes = kTile / V, kRuns = kThr / kLanes, R = kPiece / kRuns, S = kStagesOf<T, 2, V>;
    extern __shared__ __align__(16) uint8_t raw[];
    __shared__ Shared s;
    constexpr int kBytes = Stage<T, R, kWide>::kBytes;
    char* const stages = reinterpret_cast<char*>(raw);
    const unsigned tag = begin<T, 2, V, R, kThr, kWide>(g, stages, s, kBack);
    const int run = threadIdx.x / kLanes, e = threadIdx.x % kLanes * V, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int n = 0; s.ticket[n & 3] < g.total; n++) {
        if (S == 1) stage_piece<T, 2, R, kThr, kWide, true>(g, stages, s, n & 3, kBack);
        copies_wait();
        __syncthreads();
        const int drawn = draw_ticket(g);
        if (S == 2 && s.ticket[(n + 1) & 3] < g.total)
            stage_piece<T, 2, R, kThr, kWide, false>(g, stages + ((n + 1) & 1) * 2 * kBytes, s, (n + 1) & 3, kBack);
        const Piece& pc = s.piece[n & 3];
        const int tile = s.tile[n & 3], len = pc.len;
        const int staged = (S == 2 ? n & 1 : 0) * 2 * kBytes;
        const Rows<T, V, A, R, kWide> in0(staged, run, e, g.gate, g.gate_ld, pc.row0, tile * kTile);
        const Rows<T, V, A, R, kWide> in1(staged + kBytes, run, e, kBack ? g.dy : g.x, kBack ? g.dy_ld : g.x_ld, pc.row0,
                                       tile * kTile);
        F<V> a[R], b[R], P = all<V>(1.0f), H = all<V>(0.0f);
#pragma unroll
        for (int j = 0; j < R; j++) {
            F<V> keep;
            gate_pair(in0[j], a[j], keep);
            b[j] = in1[j];
            if (!kBack) b[j] = mul(b[j], keep);
        }
        if (len < kPiece) {  // steps past the end change nothing
#pragma unroll
            for (int j = 0; j < R; j++)
                if (run * R + j >= len) a[j] = all<V>(1.0f), b[j] = all<V>(0.0f);
        }
#pragma unroll
        for (int j = 0; j < R; j++) {
            P = mul(P, a[j]);
            // against time the map is built front to back: this step's dy seen through the steps before
            H = kBack ? fma(P, b[j], H) : fma(a[j], H, b[j]);
        }
#pragma unroll
        for (int i = 0; i < V; i++) s.run[run][e + i] = make_float2(P.v[i], H.v[i]);
        // where only the summary is wanted, a piece inside a group has said all with its pair
        const bool enters = (!kBack && (g.y || g.carry)) || pc.last || pc.at % kGroup == kGroup - 1;
        Looked<kThr> seen = {};
        if (enters) seen = look_back<kThr>(g, pc, tile);
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
        if (enters) settle<kThr>(g, pc, tile, seen, tag, s);
        post_ticket(g, s, (n + 2) & 3, drawn);
        __syncthreads();
        if (!enters) continue;
        if (warp == 0) {
            const float h = enter_piece(g, pc, tile, own, tag, s);
            s.enter[lane] = h;
            if (!kBack && g.carry && pc.carry >= 0 && tile * kTile + lane < g.D)
                g.carry[(int64_t)pc.carry * g.D + tile * kTile + lane] = h;
        }
        __syncthreads();
        const int ch = tile * kTile + e;
        if (!kBack && g.y && ch < g.D) {
            F<V> h;
#pragma unroll
            for (int i = 0; i < V; i++) h.v[i] = s.run[run][e + i].x * s.enter[e + i] + s.run[run][e + i].y;
            T* y = (T*)g.y + (pc.row0 + run * R) * g.y_ld + ch;
            if (len == kPiece) {
#pragma unroll
                for (int j = 0; j < R; j++, y += g.y_ld) {
                    h = fma(a[j], h, b[j]);
                    pack<T, V, A>(y, h, g.D - ch);
                }
            } else {
#pragma unroll
                for (int j = 0; j < R; j++, y += g.y_ld) {
                    h = fma(a[j], h, b[j]);
                    if (run * R + j < len) pack<T, V, A>(y, h, g.D - ch);
                }
            }
        }
    }
    finish(g);
}

// ---- backward -------------------------------------------------------------------------------------
// The states of the piece are computed again from the one that the forward pass left at its start.
template <typename T, int V, int A, bool kWide>
__global__ void __launch_bounds__(kThreads<V>, V == 4 ? 4 : 3) scan_backward_kernel(const __grid_constant__ ScanArgs g) {
    constexpr int kThr = kThreads<V>, kLanes = kTile / V, kRuns = kThr / kLanes, R = kPiece / kRuns, S = kStagesOf<T, 3, V>;
    extern __shared__ __align__(16) uint8_t raw[];
    __shared__ Shared s;
    __shared__ SharedBack sb;
    constexpr int kBytes = Stage<T, R, kWide>::kBytes;
    char* const stages = reinterpret_cast<char*>(raw);
    const unsigned tag = begin<T, 3, V, R, kThr, kWide>(g, stages, s, true);
    const int run = threadIdx.x / kLanes, e = threadIdx.x % kLanes * V, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int n = 0; s.ticket[n & 3] < g.total; n++) {
        if (S == 1) {
            __syncthreads();  // the last piece's dy has been read
            stage_piece<T, 3, R, kThr, kWide, true>(g, stages, s, n & 3, true);
        }
        copies_wait();
        __syncthreads();
        const int drawn = draw_ticket(g);
        if (S == 2 && s.ticket[(n + 1) & 3] < g.total)
            stage_piece<T, 3, R, kThr, kWide, false>(g, stages + ((n + 1) & 1) * 3 * kBytes, s, (n + 1) & 3, true);
        const Piece& pc = s.piece[n & 3];
        const int tile = s.tile[n & 3], len = pc.len;
        const int staged = (S == 2 ? n & 1 : 0) * 3 * kBytes;
        const Rows<T, V, A, R, kWide> in_g(staged, run, e, g.gate, g.gate_ld, pc.row0, tile * kTile);
        const Rows<T, V, A, R, kWide> in_x(staged + kBytes, run, e, g.x, g.x_ld, pc.row0, tile * kTile);
        const Rows<T, V, A, R, kWide> in_d(staged + 2 * kBytes, run, e, g.dy, g.dy_ld, pc.row0, tile * kTile);
        float carried = 0.0f;
        if (warp == 1 && pc.carry >= 0 && tile * kTile + lane < g.D)
            carried = g.carry[(int64_t)pc.carry * g.D + tile * kTile + lane];
        F<V> a[R], k[R], P = all<V>(1.0f), H = all<V>(0.0f), G = all<V>(0.0f);
#pragma unroll
        for (int j = 0; j < R; j++) gate_pair(in_g[j], a[j], k[j]);
        if (len < kPiece) {
#pragma unroll
            for (int j = 0; j < R; j++)
                if (run * R + j >= len) a[j] = all<V>(1.0f), k[j] = all<V>(0.0f);
        }
#pragma unroll
        for (int j = 0; j < R; j++) {
            if (run * R + j >= len) break;  // what is staged there may be anything
            P = mul(P, a[j]);
            H = fma(a[j], H, mul(k[j], in_x[j]));
            // the map of a gradient, front to back: this step's dy seen through the steps before
            G = fma(P, in_d[j], G);
        }
#pragma unroll
        for (int i = 0; i < V; i++) {
            s.run[run][e + i] = make_float2(P.v[i], G.v[i]);
            sb.hold[run][e + i] = H.v[i];
        }
        const Looked<kThr> seen = look_back<kThr>(g, pc, tile);
        __syncthreads();
        float2 own = make_float2(1.0f, 0.0f);
        if (warp == 0) {
#pragma unroll
            for (int u = kRuns - 1; u >= 0; u--) {
                const float2 p = s.run[u][lane];
                sb.after[u][lane] = own;
                own.y = p.x * own.y + p.y;
                own.x *= p.x;
            }
            publish(g.pairs + ((int64_t)pc.slot * g.tiles + tile) * kTile + lane, own.x, own.y, tag);
        }
        if (warp == 1) {  // states at the start of each run
            float h = carried;
#pragma unroll
            for (int u = 0; u < kRuns; u++) {
                const float next = s.run[u][lane].x * h + sb.hold[u][lane];
                sb.hold[u][lane] = h;
                h = next;
            }
        }
        settle<kThr>(g, pc, tile, seen, tag, s);
        post_ticket(g, s, (n + 2) & 3, drawn);
        __syncthreads();
        if (warp == 0) s.enter[lane] = enter_piece(g, pc, tile, own, tag, s);
        // (h_{t-1} - x_t) a_t (1 - a_t), while the first warp works out what enters
        F<V> f[R], h;
#pragma unroll
        for (int i = 0; i < V; i++) h.v[i] = sb.hold[run][e + i];
#pragma unroll
        for (int j = 0; j < R; j++) {
            const F<V> x = in_x[j], ak = mul(a[j], k[j]);
            f[j] = mul(fma(x, all<V>(-1.0f), h), ak);
            h = fma(a[j], h, mul(k[j], x));
        }
        __syncthreads();
        const int ch = tile * kTile + e;
        if (ch < g.D) {
            F<V> c;
#pragma unroll
            for (int i = 0; i < V; i++) c.v[i] = sb.after[run][e + i].x * s.enter[e + i] + sb.after[run][e + i].y;
            T* dg = (T*)g.dgate + (pc.row0 + run * R + R - 1) * g.dgate_ld + ch;
            T* dx = (T*)g.dx + (pc.row0 + run * R + R - 1) * g.dx_ld + ch;
#pragma unroll
            for (int j = R - 1; j >= 0; j--, dg -= g.dgate_ld, dx -= g.dx_ld) {
                if (run * R + j >= len) continue;
                const F<V> q = add(in_d[j], c);
                c = mul(a[j], q);
                pack<T, V, A>(dg, mul(f[j], q), g.D - ch);
                pack<T, V, A>(dx, mul(k[j], q), g.D - ch);
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
    F<V> a, keep, y_row = all<V>(0.0f);
    if (slot >= 0 && slot < n_slots) {
        gate_pair(unpack<T, V, V>(gate + row * gate_ld + ch), a, keep);
        y_row = fma(a, unpack<float, V, V>(state_in + slot * state_ld + ch), mul(keep, unpack<T, V, V>(x + row * x_ld + ch)));
        pack<float, V, V>(state_out + slot * state_ld + ch, y_row, V);
    }
    pack<T, V, V>(y + row * y_ld + ch, y_row, V);
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
    // CTAs per SM of the kernels used so far
    struct {
        void (*kernel)(ScanArgs);
        int per_sm;
    } fits[4] = {};

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
template <typename T, int kTensors, int V, bool kWide>
int run(sparbit_scan_plan_s* p, void (*kernel)(ScanArgs), const ScanArgs& g, cudaStream_t st) {
    constexpr int threads = kThreads<V>, R = kPiece / (threads / (kTile / V));
    constexpr size_t smem = kStagesOf<T, kTensors, V> * kTensors * Stage<T, R, kWide>::kBytes;
    auto* fit = p->fits;
    while (fit < p->fits + 3 && fit->kernel && fit->kernel != kernel) fit++;
    if (fit->kernel != kernel) {
        CU(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
        CU(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&fit->per_sm, kernel, threads, smem));
        fit->kernel = kernel;
    }
    const int most = (fit->per_sm > 0 ? fit->per_sm : 1) * p->sm_count;
    CU(launch(kernel, dim3(g.total < most ? g.total : most), dim3(threads), smem, st, g));
    return SPARBIT_OK;
}

// Calls f.template operator()<T, A>() for the plan's type and the channels an access takes.
template <typename T, int kMost, typename Fn>
int by_access(int A, Fn f) {
    if constexpr (kMost >= 4)
        if (A == 4) return f.template operator()<T, 4>();
    if (A >= 2) return f.template operator()<T, 2>();
    return f.template operator()<T, 1>();
}
template <int kMost16, int kMost32, typename Fn>
int by_type(int dtype, int A, Fn f) {
    if (dtype == SPARBIT_F32) return by_access<float, kMost32>(A, f);
    if (dtype == SPARBIT_BF16) return by_access<__nv_bfloat16, kMost16>(A, f);
    return by_access<__half, kMost16>(A, f);
}

// Channels an access takes: the most whose rows start on multiples of them, in the tensors of the
// plan's type (bits of their addresses and pitches) and in 32-bit ones.
int access_channels(int dtype, size_t D, uintptr_t bits, uintptr_t bits32) {
    const int es = (int)elem_size(dtype);
    for (int A = 4; A > 1; A /= 2)
        if (D % A == 0 && bits % (A * es) == 0 && bits32 % (A * 4) == 0) return A;
    return 1;
}

}  // namespace

extern "C" {

int sparbit_scan_plan_create(int n_seqs, const size_t* lengths, size_t channels, int dtype,
                             sparbit_scan_plan_t** out) {
    if (!out) return SPARBIT_ERR_ARG;
    *out = nullptr;
    if (!lengths || n_seqs < 1 || channels < 1 || !known_dtype(dtype)) return SPARBIT_ERR_ARG;
    if (channels > (1u << 20) || n_seqs > 65535) return SPARBIT_ERR_LIMIT;
    const size_t most = kMostElements / channels, tiles = (channels + kTile - 1) / kTile;
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
                                                 group + i / kGroup, i == n - 1, lengths[s] ? carry + q : -1, {}});
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
    for (auto& fit : p->fits) fit = {};
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
    if (bad_pitch(gate_ld, D, p->rows) || bad_pitch(x_ld, D, p->rows) || (y && bad_pitch(y_ld, D, p->rows)) ||
        (h0 && bad_pitch(h0_ld, D, p->n_seqs)))
        return SPARBIT_ERR_ARG;
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
    const uintptr_t in_bits = (uintptr_t)gate | (uintptr_t)x | gate_ld * es | x_ld * es;
    g.first = h0;
    g.first_ld = (int64_t)h0_ld;
    g.y = y;
    g.y_ld = (int64_t)y_ld;
    g.summary = summary;
    g.carry = carry;
    const int access = access_channels(p->dtype, D, in_bits | (y ? (uintptr_t)y | y_ld * es : 0), 0);
    // as many channels a thread as an access takes: 8 x 4096 x 2048 bf16 four 92 us, two 106; rows that allow only
    // single elements would be written in scattered pairs of bytes by four (8 x 8192 x 2047 409 us against 281)
    return by_type<4, 4>(p->dtype, access, [&]<typename T, int A>() {
        if constexpr (A * sizeof(T) < 16)
            if (in_bits % 16 != 0)
                return run<T, 2, A, false>(p, scan_forward_kernel<T, A, A, false, false>, g, (cudaStream_t)stream);
        return run<T, 2, A, true>(p, scan_forward_kernel<T, A, A, false, true>, g, (cudaStream_t)stream);
    });
}

int sparbit_scan_backward(sparbit_scan_plan_t* p, const void* gate, size_t gate_ld, const void* x, size_t x_ld,
                          const float* carry, const void* dy, size_t dy_ld, const float* dlast, size_t dlast_ld,
                          void* dgate, size_t dgate_ld, void* dx, size_t dx_ld, float* dsummary, void* stream) {
    if (!p || !dgate != !dx) return SPARBIT_ERR_ARG;
    const size_t D = p->D, es = elem_size(p->dtype);
    if (p->rows && (!gate || !dy || (dx && (!x || !carry)))) return SPARBIT_ERR_ARG;
    if (bad_pitch(gate_ld, D, p->rows) || bad_pitch(dy_ld, D, p->rows) || (dlast && bad_pitch(dlast_ld, D, p->n_seqs)))
        return SPARBIT_ERR_ARG;
    if (dx && (bad_pitch(x_ld, D, p->rows) || bad_pitch(dgate_ld, D, p->rows) || bad_pitch(dx_ld, D, p->rows)))
        return SPARBIT_ERR_ARG;
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
        return by_type<4, 4>(p->dtype, access_channels(p->dtype, D, in_bits, 0), [&]<typename T, int A>() {
            if constexpr (A * sizeof(T) < 16)
                if (in_bits % 16 != 0)
                    return run<T, 2, A, false>(p, scan_forward_kernel<T, A, A, true, false>, g, (cudaStream_t)stream);
            return run<T, 2, A, true>(p, scan_forward_kernel<T, A, A, true, true>, g, (cudaStream_t)stream);
        });
    }
    in_bits |= (uintptr_t)x | x_ld * es;
    g.x = x;
    g.x_ld = (int64_t)x_ld;
    g.carry = (float*)carry;
    g.dgate = dgate;
    g.dgate_ld = (int64_t)dgate_ld;
    g.dx = dx;
    g.dx_ld = (int64_t)dx_ld;
    const uintptr_t out_bits = (uintptr_t)dgate | (uintptr_t)dx | dgate_ld * es | dx_ld * es;
    // four channels a thread of 16-bit types: 8 x 4096 x 2048 bf16 162 us, with two 172 (and 8 x 8192 x 2046, whose
    // accesses take two, 444 us against 533); two of 32-bit types: 8 x 8192 x 1024 f32 238 us, with four 248; one
    // where an access takes one
    return by_type<4, 2>(p->dtype, access_channels(p->dtype, D, in_bits | out_bits, 0), [&]<typename T, int A>() {
        constexpr int V = A == 1 ? 1 : sizeof(T) == 4 ? 2 : 4;
        return in_bits % 16 == 0 ? run<T, 3, V, true>(p, scan_backward_kernel<T, V, A, true>, g, (cudaStream_t)stream)
                                 : run<T, 3, V, false>(p, scan_backward_kernel<T, V, A, false>, g, (cudaStream_t)stream);
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
    if (!slots && n_slots < rows) return SPARBIT_ERR_ARG;
    if (channels > (1u << 20) || rows > 0x7fffffffu) return SPARBIT_ERR_LIMIT;
    if (bad_pitch(gate_ld, channels, rows) || bad_pitch(x_ld, channels, rows) || bad_pitch(y_ld, channels, rows) ||
        bad_pitch(state_ld, channels, n_slots))
        return SPARBIT_ERR_ARG;
    const size_t es = elem_size(dtype);
    const Region rg{gate, rows, channels * es, gate_ld * es}, rx{x, rows, channels * es, x_ld * es},
        ry{y, rows, channels * es, y_ld * es}, rs{slots, 1, rows * 4, 0},
        ri{state_in, n_slots, channels * 4, state_ld * 4}, ro{state_out, n_slots, channels * 4, state_ld * 4};
    if (regions_overlap(ry, rg) || regions_overlap(ry, rx) || regions_overlap(ry, rs) || regions_overlap(ry, ri) ||
        regions_overlap(ry, ro) || regions_overlap(ro, rg) || regions_overlap(ro, rx) || regions_overlap(ro, rs) ||
        (state_in != state_out && regions_overlap(ro, ri)))
        return SPARBIT_ERR_ALIAS;
    const uintptr_t bits = (uintptr_t)gate | (uintptr_t)x | (uintptr_t)y | gate_ld * es | x_ld * es | y_ld * es;
    const int V = access_channels(dtype, channels, bits, (uintptr_t)state_in | (uintptr_t)state_out | state_ld * 4);
    return by_type<4, 4>(dtype, V, [&]<typename T, int kV>() {
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
    if (!gathered || !out) return SPARBIT_ERR_ARG;
    if (channels > (1u << 20) || n_ranks > 65535) return SPARBIT_ERR_LIMIT;
    if (bad_pitch(out_ld, channels, n_ranks)) return SPARBIT_ERR_ARG;
    if ((size_t)P * 2 * channels > kMostElements / n_ranks) return SPARBIT_ERR_OVERFLOW;
    const Region rg{gathered, 1, (size_t)n_ranks * P * 2 * channels * 4, 0}, rh{h0, 1, channels * 4, 0},
        ro{out, (size_t)n_ranks, channels * 4, out_ld * 4};
    if (regions_overlap(ro, rg) || regions_overlap(ro, rh)) return SPARBIT_ERR_ALIAS;
    CU(launch(scan_join_kernel, dim3((unsigned)((channels + 127) / 128), (unsigned)n_ranks), dim3(128), 0,
              (cudaStream_t)stream, P, first_rank, (int)channels, gathered, h0, out, (int64_t)out_ld, reverse));
    return SPARBIT_OK;
}

}  // extern "C"
