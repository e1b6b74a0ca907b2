// wm_seq_scan.cu -- the gated linear recurrence over time and its gradients.
//
//   keep = sigmoid(gate), write = 1 - keep;  h_t = keep_t h_{t-1} + write_t x_t
//   backward, from the last step down, with c the gradient flowing into h_t from later steps:
//   L = dh_t + c;  dx = L write;  dgate = L (h_{t-1} - x) keep write;  c = keep L
//
// Both are st -> A st + B per step (A = keep; B = write x, or keep dh), so a span of steps is
// st -> P st + S with P the product of its keeps and S its result from 0.  A span that holds a
// reset ignores what enters it, whatever that is: its P carries a minus sign, which products
// with keeps leave there, and the state is selected, not multiplied by 0 (which would keep an
// inf or NaN).  States, P and S are fp32.
//
// Bound by memory: forward reads gate and x and writes h (6 bytes a value in bf16, about 15
// instructions), backward reads gate, x, h and dh and writes two gradients (12 bytes).  Three
// kernels, each reading its inputs once:
//   k_scan_walk    T <= 8 (a dream's step): a thread walks its channels, all loads in flight.
//   k_scan_stream  enough channels to fill the GPU: a thread walks its channels over all
//                  steps, its inputs arriving in a ring in shared memory by asynchronous copies
//                  that hold no registers; every thread waits for its own copies only.
//   k_scan_spans   few channels: time is cut into spans of L steps, one per warp and all at once;
//                  a CTA joins its spans in shared memory and finds the state entering them from
//                  the (P, S) that the CTAs before it publish.  The spans' inputs stay in shared
//                  memory between the two passes.
//
// Measured (bf16, one GB300, durations of the kernels alone): 128 steps x 512 x 1024 channels 61 us
// forward and 120 us backward, 6.6 and 6.7 TB/s, nearly the rate of a copy (calls one after another: 66 and
// 126); 65,536 steps x 256 channels 37 and 61 us (2.7 and 3.3 TB/s, bound by instruction issue: 45 and 85
// a value); one step of 16 x 256 channels 4 us.
#include <type_traits>

#include "wm_seq_internal.h"

namespace {

constexpr int kThreads = 128;

template <class T>
struct ScanParams {
    long long steps;
    int N, H;
    int gpr;           // groups of VEC channels per sequence: ceil(H / VEC)
    long long groups;  // N * gpr
    seq_view<const T> gate, x, h_in, dh;
    seq_view<T> h, dgate, dx;
    const float *h0;      // what enters the first step, [N, H] (backward: dh_last), or null
    const float *h_init;  // backward: the forward's h0
    const uint8_t *reset;
    const int32_t *lengths;
    float *last;  // what leaves the last step, [N, H] (backward: dh0), or null
    int *status;
};

// keep and write without cancellation in either.
//   fp32: from exp(-|p|), which neither overflows nor cancels; the selects make saturated gates exact.
//   bf16: from exp(-p), p held at -87 (NaN stays): six instructions of the forward's 20 a value.
//   There keep is 1.6e-38, the least that the reciprocal gives (results below fp32's normal range
//   are 0), and write rounds to 1.  The hardware's exponential and reciprocal (2^-21, 2^-23) are
//   far below the inputs' precision.
template <class T>
__device__ __forceinline__ void gates(float p, float &keep, float &write) {
    if constexpr (sizeof(T) == 2) {
        float e;
        asm("max.NaN.f32 %0, %1, %2;" : "=f"(p) : "f"(p), "f"(-87.f));
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(p * -1.4426950408889634f));
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(keep) : "f"(1.f + e));
        write = e * keep;
    } else {
        const float e = expf(-fabsf(p)), s = __fdividef(1.f, 1.f + e), es = e * s;
        keep = p >= 0.f ? s : es;
        write = p >= 0.f ? es : s;
    }
}

__device__ __forceinline__ long long live_steps(const int32_t *lengths, int n, long long T, int *status) {
    if (!lengths) return T;
    const int len = lengths[n];
    if (len < 0 || len > T) seq_record(status, WM_ERR_INVALID_ARG);
    return len < 0 ? 0 : len > T ? T : len;
}

// One step of VEC channels: the outputs, and the state carried on.
template <class T, int VEC>
__device__ __forceinline__ seq_vec<T, VEC> step_fwd(const seq_vec<T, VEC> &g, const seq_vec<T, VEC> &x, bool cut,
                                                    float (&st)[VEC]) {
    float fg[VEC], fx[VEC];
    seq_unpack(g, fg);
    seq_unpack(x, fx);
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
        float keep, write;
        gates<T>(fg[k], keep, write);
        st[k] = fmaf(keep, cut ? 0.f : st[k], write * fx[k]);
    }
    return seq_pack<T, VEC>(st);
}
template <class T, int VEC>
__device__ __forceinline__ void step_bwd(const seq_vec<T, VEC> &g, const seq_vec<T, VEC> &x, const seq_vec<T, VEC> &dh,
                                         const float (&before)[VEC], bool cut, float (&c)[VEC], seq_vec<T, VEC> &dgate,
                                         seq_vec<T, VEC> &dx) {
    float fg[VEC], fx[VEC], fd[VEC];
    seq_unpack(g, fg);
    seq_unpack(x, fx);
    seq_unpack(dh, fd);
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
        float keep, write;
        gates<T>(fg[k], keep, write);
        const float L = fd[k] + c[k], lw = L * write;
        fg[k] = lw * ((cut ? 0.f : before[k]) - fx[k]) * keep;
        fx[k] = lw;
        c[k] = cut ? 0.f : keep * L;
    }
    dgate = seq_pack<T, VEC>(fg);
    dx = seq_pack<T, VEC>(fx);
}

template <int VEC>
__device__ __forceinline__ void read_state(float (&st)[VEC], const float *p, long long c) {
#pragma unroll
    for (int k = 0; k < VEC; ++k) st[k] = p ? p[c + k] : 0.f;
}
template <int VEC>
__device__ __forceinline__ void write_state(float *p, long long c, const float (&st)[VEC]) {
    if (p)
#pragma unroll
        for (int k = 0; k < VEC; ++k) p[c + k] = st[k];
}

// The outputs of padded steps [from, to).
template <class T, int VEC, bool BWD>
__device__ __forceinline__ void pad(const ScanParams<T> &a, int n, int j, long long from, long long to) {
    seq_vec<T, VEC> zero;
#pragma unroll
    for (int k = 0; k < VEC; ++k) zero.v[k] = seq_from_float<T>(0.f);
    for (long long t = from; t < to; ++t) {
        if (!BWD) {
            seq_store(a.h.row(t, n) + j, zero);
        } else {
            seq_store(a.dgate.row(t, n) + j, zero);
            seq_store(a.dx.row(t, n) + j, zero);
        }
    }
}

// ---- T <= kWalk: one thread, all steps' loads in flight together ------------------------
constexpr int kWalk = 8;

template <class T, int VEC, bool BWD>
__global__ void __launch_bounds__(kThreads) k_scan_walk(const ScanParams<T> a) {
    using V = seq_vec<T, VEC>;
    constexpr int U = VEC * sizeof(T) >= 8 ? 2 : 4;
    const long long grp = (long long)blockIdx.x * kThreads + threadIdx.x;
    if (grp >= a.groups) return;
    const int n = (int)(grp / a.gpr), j = (int)(grp - (long long)n * a.gpr) * VEC;
    const long long c = (long long)n * a.H + j;
    float st[VEC];
    read_state<VEC>(st, a.h0, c);
    const int live = (int)live_steps(a.lengths, n, a.steps, a.status);
    for (int i = 0; i < live; i += U) {
        V vg[U], vx[U], vd[U], vh[U];
        bool cut[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int t = BWD ? live - 1 - (i + u) : i + u;
            if (i + u < live) {
                vg[u] = seq_load<T, VEC>(a.gate.row(t, n) + j);
                vx[u] = seq_load<T, VEC>(a.x.row(t, n) + j);
                if (BWD) vd[u] = seq_load<T, VEC>(a.dh.row(t, n) + j);
                if (BWD && t > 0) vh[u] = seq_load<T, VEC>(a.h_in.row(t - 1, n) + j);
                cut[u] = a.reset && a.reset[(long long)t * a.N + n];
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (i + u >= live) break;
            const int t = BWD ? live - 1 - (i + u) : i + u;
            if (!BWD) {
                seq_store(a.h.row(t, n) + j, step_fwd<T, VEC>(vg[u], vx[u], cut[u], st));
            } else {
                float before[VEC];
                if (t > 0) seq_unpack(vh[u], before);
                else read_state<VEC>(before, a.h_init, c);
                V dgate, dx;
                step_bwd<T, VEC>(vg[u], vx[u], vd[u], before, cut[u], st, dgate, dx);
                seq_store(a.dgate.row(t, n) + j, dgate);
                seq_store(a.dx.row(t, n) + j, dx);
            }
        }
    }
    pad<T, VEC, BWD>(a, n, j, live, a.steps);
    write_state<VEC>(a.last, c, st);
}

// ---- many channels: a thread's inputs stream through a ring of its own -------------------
// The ring holds GROUPS groups of KG steps; a group is one set of asynchronous copies, and its
// steps are worked on together: their gates do not wait for one another, only the state does.
template <class T, int VEC, bool BWD, bool RESET, int KG, int GROUPS>
__global__ void __launch_bounds__(kThreads) k_scan_stream(const ScanParams<T> a) {
    using V = seq_vec<T, VEC>;
    constexpr int ARRAYS = BWD ? 4 : 2, BYTES = sizeof(V);
    extern __shared__ __align__(16) unsigned char ring[];  // [GROUPS * KG][ARRAYS][kThreads] of V
    const long long grp = (long long)blockIdx.x * kThreads + threadIdx.x;
    if (grp >= a.groups) return;  // (no barrier below)
    const int n = (int)(grp / a.gpr), j = (int)(grp - (long long)n * a.gpr) * VEC;
    const long long c = (long long)n * a.H + j;
    const int live = (int)live_steps(a.lengths, n, a.steps, a.status);
    float st[VEC], init[VEC];
    read_state<VEC>(st, a.h0, c);
    if (BWD) read_state<VEC>(init, a.h_init, c);
    V *const mine = reinterpret_cast<V *>(ring) + threadIdx.x;
    const uint32_t base = (uint32_t)__cvta_generic_to_shared(mine);
    // the rows of the next step to copy and of the next to write, moved by one step at a time
    const long long first = BWD ? live - 1ll : 0;
    const int dir = BWD ? -1 : 1;
    const T *pg = a.gate.row(first, n) + j, *px = a.x.row(first, n) + j;
    const T *pd = BWD ? a.dh.row(first, n) + j : nullptr, *ph = BWD ? a.h_in.row(first - 1, n) + j : nullptr;
    T *o0 = (BWD ? a.dgate.row(first, n) : a.h.row(first, n)) + j, *o1 = BWD ? a.dx.row(first, n) + j : nullptr;
    const uint8_t *pr = RESET ? a.reset + first * a.N + n : nullptr;
    const long long rn = dir * (long long)a.N;
    int ahead = 0;  // steps whose copies were issued
    auto issue = [&](int slot) {
#pragma unroll
        for (int u = 0; u < KG; ++u) {
            if (ahead < live) {
                const uint32_t to = base + (uint32_t)(slot * KG + u) * (ARRAYS * kThreads * BYTES);
                copy_async<BYTES>(to, pg);
                copy_async<BYTES>(to + kThreads * BYTES, px);
                if (BWD) {
                    copy_async<BYTES>(to + 2 * kThreads * BYTES, pd);
                    // (the first step has no row before it)
                    if (ahead + 1 < live) copy_async<BYTES>(to + 3 * kThreads * BYTES, ph);
                }
            }
            ++ahead;
            pg += dir * a.gate.st;
            px += dir * a.x.st;
            if (BWD) {
                pd -= a.dh.st;
                ph -= a.h_in.st;
            }
        }
        copy_commit();
    };
#pragma unroll
    for (int q = 0; q < GROUPS - 1; ++q) issue(q);
    int slot = 0;
    uint8_t cut_next[KG] = {};
    auto marks = [&](int i) {  // the group's that starts at step i
        if (RESET) {
#pragma unroll
            for (int u = 0; u < KG; ++u)
                if (i + u < live) cut_next[u] = pr[u * rn];
            pr += KG * rn;
        }
    };
    marks(0);
    for (int i = 0; i < live; i += KG) {
        bool cut[KG];
#pragma unroll
        for (int u = 0; u < KG; ++u) cut[u] = RESET && cut_next[u];
        marks(i + KG);
        issue(slot == 0 ? GROUPS - 1 : slot - 1);
        copy_wait<GROUPS - 1>();
        const V *r = mine + slot * KG * (ARRAYS * kThreads);
        auto step = [&](const V &g, const V &x, const V &d, const V &h, int u) {
            if (!BWD) {
                seq_store(o0, step_fwd<T, VEC>(g, x, cut[u], st));
                o0 += a.h.st;
            } else {
                float before[VEC];
                seq_unpack(h, before);
                if (i + u + 1 == live)
#pragma unroll
                    for (int k = 0; k < VEC; ++k) before[k] = init[k];
                V dgate, dx;
                step_bwd<T, VEC>(g, x, d, before, cut[u], st, dgate, dx);
                seq_store(o0, dgate);
                seq_store(o1, dx);
                o0 -= a.dgate.st;
                o1 -= a.dx.st;
            }
        };
        auto read = [&](int u, int array) { return r[(u * ARRAYS + (BWD ? array : min(array, 1))) * kThreads]; };
        if (i + KG <= live) {
            V v[KG][ARRAYS];
#pragma unroll
            for (int u = 0; u < KG; ++u)
#pragma unroll
                for (int q = 0; q < ARRAYS; ++q) v[u][q] = read(u, q);
#pragma unroll
            for (int u = 0; u < KG; ++u) step(v[u][0], v[u][1], v[u][ARRAYS - 2], v[u][ARRAYS - 1], u);
        } else {
#pragma unroll
            for (int u = 0; u < KG - 1; ++u)
                if (i + u < live) step(read(u, 0), read(u, 1), read(u, 2), read(u, 3), u);
        }
        slot = slot + 1 == GROUPS ? 0 : slot + 1;
    }
    pad<T, VEC, BWD>(a, n, j, live, a.steps);
    write_state<VEC>(a.last, c, st);
}

// ---- few channels: spans of time side by side ----------------------------------------------
// A tile is W = 32 * VEC channels of one sequence, a chunk SUBS spans of L steps of it; a CTA
// takes one (chunk, tile).  Lane l of warp q holds VEC channels of span q.  Chunks are numbered
// in the order of the recurrence; 16 make a group, 16 groups a section.  Every chunk publishes
// its (P, S), the last of a group the group's, the last of a section the state that leaves it,
// and a chunk's entering state is the section's state through the groups and then the chunks
// before it, always joined in the same tree: the same bits every time.  CTAs take their
// chunks by a ticket, so a chunk waits only for chunks that are running or done.
constexpr int kSpanThreads = 256, SUBS = kSpanThreads / 32;
constexpr int kGroupBits = 4, kGroupOf = 1 << kGroupBits;
constexpr unsigned kPolls = 1u << 20;  // a wait's limit: about a second

struct SpanWork {
    unsigned *ticket;                         // (8 bytes on: a place that nothing sets)
    // places for what is published, and no more: the last chunk of a tile publishes nothing, nor does what it ends
    unsigned long long *chunk_ps, *group_ps;  // [tile][chunks - 1][W], [tile][groups][W]
    unsigned long long *section;              // [tile][sections][W]: the state leaving it
    int chunks, groups, sections, tiles;      // chunks of a tile, groups and sections with chunks after them; tiles in all
    int tiles_per_n;
    uint32_t test_wait;                       // > 0: the first chunk polls what nothing sets
};

__device__ __forceinline__ void publish(unsigned long long *p, float2 v) {
    const unsigned x = isnan(v.x) ? 0x7fffffffu : __float_as_uint(v.x);  // (never the ones of an empty place)
    const unsigned long long b = (unsigned long long)__float_as_uint(v.y) << 32 | x;
    asm volatile("st.relaxed.gpu.global.b64 [%0], %1;" ::"l"(p), "l"(b) : "memory");
}
__device__ __forceinline__ unsigned long long peek(const unsigned long long *p) {
    unsigned long long b;
    asm volatile("ld.relaxed.gpu.global.b64 %0, [%1];" : "=l"(b) : "l"(p) : "memory");
    return b;
}
__device__ __forceinline__ bool is_set(unsigned long long b) { return (unsigned)b != 0xffffffffu; }
__device__ __forceinline__ float2 unpack(unsigned long long b) {
    return make_float2(__uint_as_float((unsigned)b), __uint_as_float((unsigned)(b >> 32)));
}

// Whether the span holds a reset (the sign of P, also of -0).
__device__ __forceinline__ bool cuts_off(float p) { return __float_as_int(p) < 0; }
// Span a, then span b.
__device__ __forceinline__ float2 join(float2 a, float2 b) {
    return cuts_off(b.x) ? b : make_float2(a.x * b.x, fmaf(b.x, a.y, b.y));
}
// The state after a span.
__device__ __forceinline__ float through(float2 ps, float st) { return cuts_off(ps.x) ? ps.y : fmaf(ps.x, st, ps.y); }

// Up to MOST published spans of this thread's channel: `ask` issues the reads, `joined` waits for
// what was not there yet and joins them.  Bounded: the first wait that gives up says so in
// status[1], which the others look at now and then, and the value counts as a span of nothing.
template <int MOST>
struct Published {
    unsigned long long b[MOST];
    __device__ __forceinline__ void ask(const unsigned long long *p, int stride, int count) {
#pragma unroll
        for (int q = 0; q < MOST; ++q) b[q] = q < count ? peek(p + q * stride) : 0;
    }
    __device__ __forceinline__ float2 joined(const unsigned long long *p, int stride, int count, int *status) {
        float2 v = make_float2(1.f, 0.f);
        unsigned polls = 0;
#pragma unroll
        for (int q = 0; q < MOST; ++q) {
            if (q >= count) break;
            while (!is_set(b[q])) {
                ++polls;
                if (polls >= kPolls || (polls % 8192 == 0 && *(volatile int *)(status + 1))) {
                    seq_record(status + 1, WM_ERR_TIMEOUT);
                    b[q] = 0x3f800000ull;
                    break;
                }
                b[q] = peek(p + q * stride);
            }
            v = join(v, unpack(b[q]));
        }
        return v;
    }
};

// DEEP: more than one chunk per tile.  Logical step i is t = i, or T - 1 - i backward.
//
// The inputs wait in shared memory, every thread's in places of its own, while the chunk's (P, S)
// goes out and the state entering it comes in, and the gates are formed again for the outputs:
// six more instructions a value, but 64 registers a thread and so twice the CTAs.  (With the
// gates kept in registers, 2 CTAs an SM, a chunk took 9,300 cycles, two thirds of it spent
// waiting; 65,536 x 256 forward took 50 us.)
template <class T, int VEC, int L, bool BWD, bool RESET, bool DEEP>
__global__ void __launch_bounds__(kSpanThreads, 4) k_scan_spans(const ScanParams<T> a, const SpanWork wk) {
    using V = seq_vec<T, VEC>;
    constexpr int W = 32 * VEC, PARTS = kSpanThreads / W, EACH = kGroupOf / PARTS, ARRAYS = BWD ? 4 : 2;
    constexpr int GATE = 0, X = 1, DH = 2, HB = 3;
    constexpr bool ASYNC = sizeof(V) >= 4;
    extern __shared__ __align__(16) unsigned char held[];  // [L][ARRAYS][kSpanThreads] of V
    __shared__ float2 spans[SUBS][W], near[DEEP ? PARTS : 1][W], far[DEEP ? PARTS : 1][W];
    __shared__ float enter[W];
    __shared__ unsigned s_ticket;
    unsigned ticket = blockIdx.x;
    if (DEEP) {
        if (threadIdx.x == 0) s_ticket = atomicAdd(wk.ticket, 1u) + 1u;  // (starts at ~0)
        __syncthreads();
        ticket = s_ticket;
    }
    const int chunk = DEEP ? (int)(ticket / (unsigned)wk.tiles) : 0, tile = (int)(ticket - (unsigned)chunk * (unsigned)wk.tiles);
    const int lane = threadIdx.x % 32, sub = threadIdx.x / 32, dir = BWD ? -1 : 1;
    const int n = tile / wk.tiles_per_n, j0 = (tile - n * wk.tiles_per_n) * W, j = j0 + lane * VEC;
    const bool mine = j < a.H;
    const long long c = (long long)n * a.H + j;
    const int T_ = (int)a.steps, live = (int)live_steps(a.lengths, n, a.steps, a.status);
    const long long i0 = ((long long)chunk * SUBS + sub) * L, t0 = BWD ? T_ - 1 - i0 : i0;
    // the span's steps u in [0, steps) exist, and those in [skip, count) are not padding
    const int steps = (int)max(0ll, min((long long)L, T_ - i0));
    const int skip = BWD ? (int)max(0ll, min((long long)L, t0 - live + 1)) : 0;
    const int count = mine ? BWD ? steps : (int)max(0ll, min((long long)L, live - i0)) : 0;
    V *const own_v = reinterpret_cast<V *>(held) + threadIdx.x;
    auto at = [&](int u, int array) -> V & { return own_v[(u * ARRAYS + array) * kSpanThreads]; };
    {
        const T *pg = a.gate.row(t0, n) + j, *px = a.x.row(t0, n) + j;
        const T *pd = BWD ? a.dh.row(t0, n) + j : nullptr, *ph = BWD ? a.h_in.row(t0 - 1, n) + j : nullptr;
        auto bring = [&](int u, int array, const T *p) {
            if constexpr (ASYNC) copy_async<(int)sizeof(V)>((uint32_t)__cvta_generic_to_shared(&at(u, array)), p);
            else at(u, array) = seq_load<T, VEC>(p);
        };
#pragma unroll
        for (int u = 0; u < L; ++u) {
            if (u >= skip && u < count) {
                bring(u, GATE, pg);
                bring(u, X, px);
                if (BWD) {
                    bring(u, DH, pd);
                    if (t0 > u) bring(u, HB, ph);
                }
            }
            pg += dir * a.gate.st;
            px += dir * a.x.st;
            if (BWD) {
                pd -= a.dh.st;
                ph -= a.h_in.st;
            }
        }
        if (ASYNC) copy_commit();
    }
    unsigned cuts = 0;
    if (RESET) {  // lane u has step u's
        const bool in = lane >= skip && lane < (BWD ? steps : (int)min((long long)L, live - i0));
        cuts = __ballot_sync(0xffffffffu, in && a.reset[(t0 + dir * lane) * a.N + n] != 0);
    }
    float P[VEC], S[VEC];
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
        P[k] = 1.f;
        S[k] = 0.f;
    }
    if (ASYNC) copy_wait<0>();
#pragma unroll 4
    for (int u = skip; u < count; ++u) {
        const bool cut = RESET && (cuts >> u & 1);
        float g[VEC], y[VEC];
        seq_unpack(at(u, GATE), g);
        seq_unpack(at(u, BWD ? DH : X), y);
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
            float keep, write;
            gates<T>(g[k], keep, write);
            if (!BWD) S[k] = fmaf(keep, cut ? 0.f : S[k], write * y[k]);
            else S[k] = cut ? 0.f : keep * (y[k] + S[k]);
            P[k] = cut ? -1.f : P[k] * keep;
        }
    }
#pragma unroll
    for (int k = 0; k < VEC; ++k) spans[sub][lane * VEC + k] = make_float2(P[k], S[k]);
    __syncthreads();
    // a thread per channel and part from here on
    const int ch = threadIdx.x % W, part = threadIdx.x / W;
    const bool more = chunk + 1 < wk.chunks;
    float2 own = make_float2(1.f, 0.f);
    if (part == 0) {
        float2 v[SUBS];
#pragma unroll
        for (int q = 0; q < SUBS; ++q) v[q] = spans[q][ch];
#pragma unroll
        for (int q = 0; q < SUBS; ++q) {
            spans[q][ch] = own;  // from here on: what comes before the span
            own = join(own, v[q]);
        }
    }
    if (DEEP) {
        const int group = chunk >> kGroupBits, in_group = chunk & (kGroupOf - 1);
        const int section = group >> kGroupBits, in_section = group & (kGroupOf - 1);
        unsigned long long *cp = wk.chunk_ps + ((long long)tile * (wk.chunks - 1) + group * kGroupOf) * W + ch;
        unsigned long long *gp = wk.group_ps + ((long long)tile * wk.groups + section * kGroupOf) * W + ch;
        unsigned long long *sp = wk.section + ((long long)tile * wk.sections + section) * W + ch;
        // h0 is read before the chunk publishes: `last` may be the same array, and the last chunk writes it
        // once all have published
        float st = 0.f;
        if (part == 0) {
            if (section == 0 && j0 + ch < a.H && a.h0) {
                st = *(const volatile float *)(a.h0 + (long long)n * a.H + j0 + ch);
                if (a.h0 == a.last) __threadfence();
            }
            if (more) publish(cp + in_group * W, own);
        }
        if (wk.test_wait && ticket == 0 && threadIdx.x == 0) {
            unsigned left = wk.test_wait;
            while (!is_set(peek(reinterpret_cast<unsigned long long *>(wk.ticket) + 1)) && left-- > 0) {}
            seq_record(a.status + 1, WM_ERR_TIMEOUT);
        }
        const int from = part * EACH, n_near = min(EACH, in_group - from), n_far = min(EACH, in_section - from);
        Published<EACH> pub;
        unsigned long long s0 = 0;
        if (in_group) pub.ask(cp + from * W, W, n_near);
        if (part == 0 && section > 0) s0 = peek(sp - W);
        if (in_group) {
            near[part][ch] = pub.joined(cp + from * W, W, n_near, a.status);
            if (in_group == kGroupOf - 1 && more) {  // the group's (P, S) goes out before anything else is waited for
                __syncthreads();
                if (part == 0) {
                    float2 v = near[0][ch];
#pragma unroll
                    for (int q = 1; q < PARTS; ++q) v = join(v, near[q][ch]);
                    publish(gp + in_section * W, join(v, own));
                }
            }
        }
        if (in_section) {
            pub.ask(gp + from * W, W, n_far);
            far[part][ch] = pub.joined(gp + from * W, W, n_far, a.status);
        }
        __syncthreads();
        if (part == 0) {
            if (section > 0) {
                Published<1> left{{s0}};
                st = left.joined(sp - W, 0, 1, a.status).y;
            }
            if (in_section)
#pragma unroll
                for (int q = 0; q < PARTS; ++q) st = through(far[q][ch], st);
            if (in_group)
#pragma unroll
                for (int q = 0; q < PARTS; ++q) st = through(near[q][ch], st);
            enter[ch] = st;
            st = through(own, st);
            if (more && in_group == kGroupOf - 1 && in_section == kGroupOf - 1) publish(sp, make_float2(0.f, st));
            if (!more && a.last && j0 + ch < a.H) a.last[(long long)n * a.H + j0 + ch] = st;
        }
    } else if (part == 0) {
        const float st = j0 + ch < a.H && a.h0 ? a.h0[(long long)n * a.H + j0 + ch] : 0.f;
        enter[ch] = st;
        if (a.last && j0 + ch < a.H) a.last[(long long)n * a.H + j0 + ch] = through(own, st);
    }
    __syncthreads();
    // the outputs, from the state entering the span
    float mid[VEC];
#pragma unroll
    for (int k = 0; k < VEC; ++k) mid[k] = through(spans[sub][lane * VEC + k], enter[lane * VEC + k]);
    T *o0 = (BWD ? a.dgate.row(t0, n) : a.h.row(t0, n)) + j, *o1 = BWD ? a.dx.row(t0, n) + j : nullptr;
    const long long d0 = dir * (BWD ? a.dgate.st : a.h.st);
    const V zero = [] {
        V z;
#pragma unroll
        for (int k = 0; k < VEC; ++k) z.v[k] = seq_from_float<T>(0.f);
        return z;
    }();
    for (int u = 0; u < (mine ? skip : 0); ++u) {  // (backward only)
        seq_store(o0, zero);
        seq_store(o1, zero);
        o0 += d0;
        o1 -= a.dx.st;
    }
#pragma unroll 4
    for (int u = skip; u < count; ++u) {
        const bool cut = RESET && (cuts >> u & 1);
        if (!BWD) {
            seq_store(o0, step_fwd<T, VEC>(at(u, GATE), at(u, X), cut, mid));
        } else {
            float before[VEC];
            if (t0 > u) seq_unpack(at(u, HB), before);
            else read_state<VEC>(before, a.h_init, c);
            V dgate, dx;
            step_bwd<T, VEC>(at(u, GATE), at(u, X), at(u, DH), before, cut, mid, dgate, dx);
            seq_store(o0, dgate);
            seq_store(o1, dx);
            o1 -= a.dx.st;
        }
        o0 += d0;
    }
    if (!BWD)
        for (int u = count; u < (mine ? steps : 0); ++u) {
            seq_store(o0, zero);
            o0 += d0;
        }
}

__global__ void k_scan_state(long long C, const float *h0, float *last) {
    const long long c = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    if (c < C) last[c] = h0 ? h0[c] : 0.f;
}

// The most values per access, `most` or a half, a quarter ... of it, that alignment, strides and H allow.
int width(const seq_scan_args &a, bool bwd, int most) {
    const size_t es = a.dtype == WM_BF16 ? 2 : 4;
    auto ok = [&](const wm_seq_view &v, int w) {
        return (uintptr_t)v.data % (w * es) == 0 && v.stride_t % w == 0 && v.stride_n % w == 0;
    };
    auto fits = [&](int w) {
        return a.H % w == 0 && ok(a.gate, w) && ok(a.x, w) && ok(a.h, w) &&
               (!bwd || (ok(a.dh, w) && ok(a.dgate, w) && ok(a.dx, w)));
    };
    while (most > 1 && !fits(most)) most /= 2;
    return most;
}

template <class T>
ScanParams<T> params(const wm_seq *h, const seq_scan_args &a, int vec, bool bwd) {
    ScanParams<T> q{};
    q.steps = a.T; q.N = a.N; q.H = a.H;
    q.gpr = (a.H + vec - 1) / vec; q.groups = (long long)a.N * q.gpr;
    auto in = [](const wm_seq_view &v) { return seq_view<const T>{(const T *)v.data, v.stride_t, v.stride_n}; };
    auto out = [](const wm_seq_view &v) { return seq_view<T>{(T *)v.data, v.stride_t, v.stride_n}; };
    q.gate = in(a.gate); q.x = in(a.x);
    if (bwd) {
        q.h_in = in(a.h); q.dh = in(a.dh); q.dgate = out(a.dgate); q.dx = out(a.dx);
        q.h0 = a.dh_last; q.h_init = a.h0; q.last = a.dh0;
    } else {
        q.h = out(a.h); q.h0 = a.h0; q.last = a.h_last;
    }
    q.reset = a.reset; q.lengths = a.lengths; q.status = h->status;
    return q;
}

unsigned blocks(long long groups) { return (unsigned)((groups + kThreads - 1) / kThreads); }

template <class T, int VEC, bool BWD>
cudaError_t walk(const wm_seq *h, const seq_scan_args &a, cudaStream_t s) {
    const ScanParams<T> q = params<T>(h, a, VEC, BWD);
    k_scan_walk<T, VEC, BWD><<<blocks(q.groups), kThreads, 0, s>>>(q);
    return cudaGetLastError();
}

template <class T, int VEC, bool BWD, bool RESET, int KG, int GROUPS>
cudaError_t stream_launch(const ScanParams<T> &q, size_t step, cudaStream_t s) {
    auto *k = k_scan_stream<T, VEC, BWD, RESET, KG, GROUPS>;
    const size_t smem = KG * GROUPS * step;
    if (smem > 40 << 10) {
        const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
    }
    k<<<blocks(q.groups), kThreads, smem, s>>>(q);
    return cudaGetLastError();
}

// A ring of 24 steps where all CTAs run at once with it, else of 12.  (512 x 1024 channels, bf16,
// calls of the backward: 125 us with 12 steps and two CTAs an SM, 129 us with 6 steps and all at once.)
template <class T, int VEC, bool BWD>
cudaError_t stream(const wm_seq *h, const seq_scan_args &a, cudaStream_t s) {
    const ScanParams<T> q = params<T>(h, a, VEC, BWD);
    const size_t step = (BWD ? 4 : 2) * VEC * sizeof(T) * kThreads;
    const size_t per_sm = (blocks(q.groups) + h->sms - 1) / h->sms;
    const bool deep = per_sm * (24 * step + 1024) <= (size_t)224 << 10;
    auto go = [&](auto reset) {
        constexpr bool R = decltype(reset)::value;
        return deep ? stream_launch<T, VEC, BWD, R, 4, 6>(q, step, s) : stream_launch<T, VEC, BWD, R, 4, 3>(q, step, s);
    };
    return a.reset ? go(std::true_type{}) : go(std::false_type{});
}

constexpr int kLenFwd = 16, kLenBwd = 8, kLenShort = 4;
struct Plan {
    enum Kind { WALK, STREAM, SPANS } kind;
    int vec, len;
    SpanWork wk;  // (its pointers are set at the launch)
    size_t ws;
};

Plan plan(const wm_seq *h, const seq_scan_args &a, bool bwd) {
    Plan p{};
    const int w4 = a.dtype == WM_BF16 ? 2 : 1;  // values in 4 bytes
    const long long C = (long long)a.N * a.H;
    // 16-byte accesses where they leave an SM's 8 warps and more (calls of 512 x 1024 channels, bf16, no lengths: 66
    // and 125 us against 76 and 145 with 8 bytes; 200 x 512: 78 and 151 against 70 and 128)
    p.vec = width(a, bwd, C >= h->sms * 1200ll && a.T > kWalk ? 4 * w4 : 2 * w4);
    if (a.T <= kWalk) {
        p.kind = Plan::WALK;
    } else if (p.vec >= w4 && C >= (long long)h->sms * 300) {
        p.kind = Plan::STREAM;
    } else {
        p.kind = Plan::SPANS;
        if (p.vec > w4) p.vec = w4;  // rows of 128 bytes: wider tiles have shorter spans for the same room
        const int W = 32 * p.vec;
        SpanWork &k = p.wk;
        k.tiles_per_n = (a.H + W - 1) / W;
        k.tiles = a.N * k.tiles_per_n;
        // spans as long as four CTAs an SM have room for; short ones when those leave SMs idle
        p.len = bwd ? kLenBwd : kLenFwd;
        if ((a.T + SUBS * p.len - 1) / (SUBS * p.len) * k.tiles < h->sms) p.len = kLenShort;
        k.chunks = (int)((a.T + SUBS * p.len - 1) / (SUBS * p.len));
        k.groups = (k.chunks - 1) / kGroupOf;
        k.sections = k.groups / kGroupOf;
        if (k.chunks > 1) p.ws = 256 + (size_t)k.tiles * W * 8 * (k.chunks - 1ll + k.groups + k.sections);
    }
    return p;
}

template <class T, int VEC, int L, bool BWD>
cudaError_t spans(wm_seq *h, const seq_scan_args &a, const Plan &p, cudaStream_t s) {
    const ScanParams<T> q = params<T>(h, a, VEC, BWD);
    SpanWork wk = p.wk;
    const bool deep = wk.chunks > 1;
    if (deep) {
        const size_t t = (size_t)wk.tiles * 32 * VEC;
        wk.ticket = (unsigned *)h->ws;
        wk.chunk_ps = (unsigned long long *)((char *)h->ws + 256);
        wk.group_ps = wk.chunk_ps + t * (wk.chunks - 1);
        wk.section = wk.group_ps + t * wk.groups;
        wk.test_wait = h->test_wait;
        h->test_wait = 0;
        const cudaError_t e = cudaMemsetAsync(h->ws, 0xff, p.ws, s);
        if (e != cudaSuccess) return e;
    }
    auto *k = a.reset ? (deep ? k_scan_spans<T, VEC, L, BWD, true, true> : k_scan_spans<T, VEC, L, BWD, true, false>)
                      : (deep ? k_scan_spans<T, VEC, L, BWD, false, true> : k_scan_spans<T, VEC, L, BWD, false, false>);
    using V = seq_vec<T, VEC>;
    const size_t smem = (size_t)L * (BWD ? 4 : 2) * kSpanThreads * sizeof(V);
    if (smem > 24 << 10) {
        const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
    }
    k<<<(unsigned)((long long)wk.tiles * wk.chunks), kSpanThreads, smem, s>>>(q, wk);
    return cudaGetLastError();
}

template <class T, bool BWD>
cudaError_t dispatch(wm_seq *h, const seq_scan_args &a, cudaStream_t s) {
    constexpr int W4 = 4 / sizeof(T);
    const Plan p = plan(h, a, BWD);
    if (p.kind == Plan::WALK)
        return p.vec == 2 * W4 ? walk<T, 2 * W4, BWD>(h, a, s) : p.vec == W4 ? walk<T, W4, BWD>(h, a, s) : walk<T, 1, BWD>(h, a, s);
    if (p.kind == Plan::STREAM)
        return p.vec == 4 * W4 ? stream<T, 4 * W4, BWD>(h, a, s) : p.vec == 2 * W4 ? stream<T, 2 * W4, BWD>(h, a, s) : stream<T, W4, BWD>(h, a, s);
    constexpr int LONG = BWD ? kLenBwd : kLenFwd;
    if (p.vec == W4) return p.len == LONG ? spans<T, W4, LONG, BWD>(h, a, p, s) : spans<T, W4, kLenShort, BWD>(h, a, p, s);
    return p.len == LONG ? spans<T, 1, LONG, BWD>(h, a, p, s) : spans<T, 1, kLenShort, BWD>(h, a, p, s);
}

}  // namespace

size_t wm_seq_scan_ws(const wm_seq *h, const seq_scan_args &a, bool backward) { return a.T ? plan(h, a, backward).ws : 0; }

cudaError_t wm_seq_scan_launch(wm_seq *h, const seq_scan_args &a, bool backward, cudaStream_t s) {
    h->last_launches = 0;
    if (a.T == 0) {  // the state goes through
        float *last = backward ? a.dh0 : a.h_last;
        if (last) {
            const long long C = (long long)a.N * a.H;
            k_scan_state<<<(unsigned)((C + 255) / 256), 256, 0, s>>>(C, backward ? a.dh_last : a.h0, last);
            h->last_launches = 1;
        }
        return cudaGetLastError();
    }
    h->last_launches = 1;
    if (a.dtype == WM_BF16) return backward ? dispatch<__nv_bfloat16, true>(h, a, s) : dispatch<__nv_bfloat16, false>(h, a, s);
    return backward ? dispatch<float, true>(h, a, s) : dispatch<float, false>(h, a, s);
}
