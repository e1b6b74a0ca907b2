// wm_seq_scan.cu -- the gated linear recurrence over time and its gradients.
//
//   keep = sigmoid(gate), write = 1 - keep;  h_t = keep_t h_{t-1} + write_t x_t
//   backward, from the last step down, with c the gradient flowing into h_t from later steps:
//   L = dh_t + c;  dx = L write;  dgate = L (h_{t-1} - x) keep write;  c = keep L
//
// Both are st -> A st + B per step (A = keep; B = write x, or keep dh), so a span of steps is
// st -> P st + S with P the product of its keeps and S its result from 0.  A span that holds a
// reset ignores what enters it, whatever that is: P = SEQ_CUT, and the state is selected, not
// multiplied by 0 (which would keep an inf or NaN).  States, P and S are fp32.
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
//                  the (P, S) that the CTAs before it publish.  The spans' gates and values stay
//                  in registers between the two passes.
#include <type_traits>

#include "wm_seq_internal.h"

namespace {

constexpr float SEQ_CUT = -1.f;  // P of a span with a reset inside (products of keeps are >= 0)
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
template <class T>
__device__ __forceinline__ void gates(float p, float &keep, float &write) {
    // bf16 inputs: the hardware exponential's relative error (about 2^-21) is far below the inputs'
    const float e = sizeof(T) == 2 ? __expf(-fabsf(p)) : expf(-fabsf(p));
    const float s = __fdividef(1.f, 1.f + e), es = e * s;
    keep = p >= 0.f ? s : es;
    write = p >= 0.f ? es : s;
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
    seq_vec<T, VEC> o;
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
        float keep, write;
        gates<T>(seq_to_float(g.v[k]), keep, write);
        st[k] = fmaf(keep, cut ? 0.f : st[k], write * seq_to_float(x.v[k]));
        o.v[k] = seq_from_float<T>(st[k]);
    }
    return o;
}
template <class T, int VEC>
__device__ __forceinline__ void step_bwd(const seq_vec<T, VEC> &g, const seq_vec<T, VEC> &x, const seq_vec<T, VEC> &dh,
                                         const float (&before)[VEC], bool cut, float (&c)[VEC], seq_vec<T, VEC> &dgate,
                                         seq_vec<T, VEC> &dx) {
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
        float keep, write;
        gates<T>(seq_to_float(g.v[k]), keep, write);
        const float L = seq_to_float(dh.v[k]) + c[k];
        dgate.v[k] = seq_from_float<T>(L * ((cut ? 0.f : before[k]) - seq_to_float(x.v[k])) * keep * write);
        dx.v[k] = seq_from_float<T>(L * write);
        c[k] = cut ? 0.f : keep * L;
    }
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
                if (t > 0)
#pragma unroll
                    for (int k = 0; k < VEC; ++k) before[k] = seq_to_float(vh[u].v[k]);
                else
                    read_state<VEC>(before, a.h_init, c);
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
// The ring holds GROUPS groups of kGroup steps; a group is one set of asynchronous copies.
constexpr int kGroup = 2;

template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t dst, const void *src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

template <class T, int VEC, bool BWD, bool RESET, int GROUPS>
__global__ void __launch_bounds__(kThreads) k_scan_stream(const ScanParams<T> a) {
    using V = seq_vec<T, VEC>;
    constexpr int ARRAYS = BWD ? 4 : 2, BYTES = sizeof(V);
    extern __shared__ __align__(16) unsigned char ring[];  // [GROUPS * kGroup][ARRAYS][kThreads] of V
    const long long grp = (long long)blockIdx.x * kThreads + threadIdx.x;
    if (grp >= a.groups) return;  // (no barrier below)
    const int n = (int)(grp / a.gpr), j = (int)(grp - (long long)n * a.gpr) * VEC;
    const long long c = (long long)n * a.H + j;
    const long long live = live_steps(a.lengths, n, a.steps, a.status);
    float st[VEC];
    read_state<VEC>(st, a.h0, c);
    V *const mine = reinterpret_cast<V *>(ring) + threadIdx.x;
    const uint32_t base = (uint32_t)__cvta_generic_to_shared(mine);
    // the rows of the next step to copy and of the next to write, moved by one step at a time
    const long long first = BWD ? live - 1 : 0;
    const int dir = BWD ? -1 : 1;
    const T *pg = a.gate.row(first, n) + j, *px = a.x.row(first, n) + j;
    const T *pd = BWD ? a.dh.row(first, n) + j : nullptr, *ph = BWD ? a.h_in.row(first - 1, n) + j : nullptr;
    T *o0 = (BWD ? a.dgate.row(first, n) : a.h.row(first, n)) + j, *o1 = BWD ? a.dx.row(first, n) + j : nullptr;
    const uint8_t *pr = RESET ? a.reset + first * a.N + n : nullptr;
    long long ahead = 0;  // steps whose copies were issued
    auto issue = [&](int slot) {
#pragma unroll
        for (int u = 0; u < kGroup; ++u) {
            if (ahead < live) {
                const uint32_t to = base + (uint32_t)(slot * kGroup + u) * (ARRAYS * kThreads * BYTES);
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
    uint8_t cut_next[kGroup] = {};
    if (RESET)
#pragma unroll
        for (int u = 0; u < kGroup; ++u)
            if (u < live) cut_next[u] = pr[u * dir * (long long)a.N];
    for (long long i = 0; i < live; i += kGroup) {
        uint8_t cut[kGroup];
#pragma unroll
        for (int u = 0; u < kGroup; ++u) cut[u] = cut_next[u];
        if (RESET) {
            pr += kGroup * dir * (long long)a.N;
#pragma unroll
            for (int u = 0; u < kGroup; ++u)
                if (i + kGroup + u < live) cut_next[u] = pr[u * dir * (long long)a.N];
        }
        issue(slot == 0 ? GROUPS - 1 : slot - 1);
        copy_wait<GROUPS - 1>();
#pragma unroll
        for (int u = 0; u < kGroup; ++u) {
            if (i + u >= live) break;
            const V *r = mine + (slot * kGroup + u) * (ARRAYS * kThreads);
            const bool ct = RESET && cut[u];
            if (!BWD) {
                seq_store(o0, step_fwd<T, VEC>(r[0], r[kThreads], ct, st));
                o0 += a.h.st;
            } else {
                float before[VEC];
                if (i + u + 1 < live) {
                    const V vh = r[3 * kThreads];
#pragma unroll
                    for (int k = 0; k < VEC; ++k) before[k] = seq_to_float(vh.v[k]);
                } else {
                    read_state<VEC>(before, a.h_init, c);
                }
                V dgate, dx;
                step_bwd<T, VEC>(r[0], r[kThreads], r[2 * kThreads], before, ct, st, dgate, dx);
                seq_store(o0, dgate);
                seq_store(o1, dx);
                o0 -= a.dgate.st;
                o1 -= a.dx.st;
            }
        }
        slot = slot + 1 == GROUPS ? 0 : slot + 1;
    }
    pad<T, VEC, BWD>(a, n, j, live, a.steps);
    write_state<VEC>(a.last, c, st);
}

// ---- few channels: spans of time side by side ----------------------------------------------
// A tile is W = 32 * VEC channels of one sequence, a chunk SUBS spans of L steps of it; a CTA
// takes one (chunk, tile).  Lane l of warp q holds VEC channels of span q.  Chunks are numbered
// in the order of the recurrence; 32 make a group, 32 groups a section.  Every chunk publishes
// its (P, S), the last of a group the group's, the last of a section the state that leaves it,
// and a chunk's entering state is the section's state through the groups and then the chunks
// before it, always joined in the same tree: the same bits every time.  CTAs take their
// chunks by a ticket, so a chunk waits only for chunks that are running or done.
constexpr int kSpanThreads = 256, SUBS = kSpanThreads / 32;
constexpr unsigned kPolls = 1u << 20;  // a wait's limit: about a second
constexpr unsigned long long kUnset = ~0ull;

struct SpanWork {
    unsigned *ticket;
    unsigned long long *chunk_ps, *group_ps;  // [tile][groups][W][32], [tile][sections][W][32]
    unsigned long long *section;              // [tile][sections][W]: the state entering it
    int chunks, groups, sections, tiles;      // chunks, groups, sections of a tile; tiles in all
    int tiles_per_n;
    uint32_t test_wait;                       // > 0: the first chunk polls what nothing sets
};

__device__ __forceinline__ void publish(unsigned long long *p, float2 v) {
    const unsigned x = isnan(v.x) ? 0x7fffffffu : __float_as_uint(v.x);  // (never kUnset)
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

// Span a, then span b.
__device__ __forceinline__ float2 join(float2 a, float2 b) {
    if (b.x < 0.f) return b;
    return make_float2(a.x < 0.f ? a.x : a.x * b.x, fmaf(b.x, a.y, b.y));
}
// The state after a span.
__device__ __forceinline__ float through(float2 ps, float st) { return ps.x < 0.f ? ps.y : fmaf(ps.x, st, ps.y); }

// Lanes' spans joined in lane order; lane 0 has the result.
__device__ __forceinline__ float2 join_lanes(float2 v) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const float2 w = make_float2(__shfl_down_sync(0xffffffffu, v.x, o), __shfl_down_sync(0xffffffffu, v.y, o));
        v = join(v, w);
    }
    return v;
}

// Polls until every lane's value is there.  Bounded: the first wait that gives up says so in
// status[1], which the others look at now and then, and the value counts as a span of nothing.
__device__ __forceinline__ float2 wait_for(unsigned long long b, const unsigned long long *p, bool want, int *status) {
    unsigned polls = 0;
    while (!__all_sync(0xffffffffu, !want || is_set(b))) {
        ++polls;
        if (polls == kPolls || (polls % 8192 == 0 && *(volatile int *)(status + 1))) {
            if (threadIdx.x % 32 == 0) seq_record(status + 1, WM_ERR_TIMEOUT);
            break;
        }
        if (want) b = peek(p);
    }
    return want && is_set(b) ? unpack(b) : make_float2(1.f, 0.f);
}

// SPANS > 1 chunk per tile: DEEP.  Logical step i is t = i, or T - 1 - i backward.
template <class T, int VEC, int L, bool BWD, bool RESET, bool DEEP>
__global__ void __launch_bounds__(kSpanThreads, 2) k_scan_spans(const ScanParams<T> a, const SpanWork wk) {
    using V = seq_vec<T, VEC>;
    constexpr int W = 32 * VEC, PER_WARP = W / SUBS;
    __shared__ float2 spans[SUBS][W], whole[W];
    __shared__ float enter[W];
    __shared__ unsigned s_ticket;
    unsigned ticket = blockIdx.x;
    if (DEEP) {
        if (threadIdx.x == 0) s_ticket = atomicAdd(wk.ticket, 1u) + 1u;  // (starts at ~0)
        __syncthreads();
        ticket = s_ticket;
    }
    const int chunk = DEEP ? (int)(ticket / (unsigned)wk.tiles) : 0, tile = (int)(ticket - (unsigned)chunk * (unsigned)wk.tiles);
    const int lane = threadIdx.x % 32, sub = threadIdx.x / 32;
    const int n = tile / wk.tiles_per_n, j0 = (tile - n * wk.tiles_per_n) * W, j = j0 + lane * VEC;
    const bool mine = j < a.H;
    const long long c = (long long)n * a.H + j, T_ = a.steps;
    const long long live = live_steps(a.lengths, n, T_, a.status);
    const long long i0 = ((long long)chunk * SUBS + sub) * L, t0 = BWD ? T_ - 1 - i0 : i0;
    const int dir = BWD ? -1 : 1;

    // per step: A and B, and what the second pass takes besides
    float A[L][VEC], B[L][VEC], wr[BWD ? L : 1][VEC], df[BWD ? L : 1][VEC];
    float2 ps[VEC];
#pragma unroll
    for (int k = 0; k < VEC; ++k) ps[k] = make_float2(1.f, 0.f);
    unsigned cuts = 0;
    {
        V rg[L], rx[L], rd[BWD ? L : 1], rh[BWD ? L : 1];
        const T *pg = a.gate.row(t0, n) + j, *px = a.x.row(t0, n) + j;
        const T *pd = BWD ? a.dh.row(t0, n) + j : nullptr, *ph = BWD ? a.h_in.row(t0 - 1, n) + j : nullptr;
#pragma unroll
        for (int u = 0; u < L; ++u) {
            const long long t = BWD ? t0 - u : t0 + u;
            if (mine && t >= 0 && t < live) {
                rg[u] = seq_load<T, VEC>(pg);
                rx[u] = seq_load<T, VEC>(px);
                if (BWD) rd[u] = seq_load<T, VEC>(pd);
                if (BWD && t > 0) rh[u] = seq_load<T, VEC>(ph);
            }
            pg += dir * a.gate.st;
            px += dir * a.x.st;
            if (BWD) {
                pd -= a.dh.st;
                ph -= a.h_in.st;
            }
        }
        if (RESET) {  // lane u has step u's
            const long long t = BWD ? t0 - lane : t0 + lane;
            cuts = __ballot_sync(0xffffffffu, lane < L && t >= 0 && t < live && a.reset[t * a.N + n] != 0);
        }
#pragma unroll
        for (int u = 0; u < L; ++u) {
            const long long t = BWD ? t0 - u : t0 + u;
            const bool in = mine && t >= 0 && t < live, cut = RESET && (cuts >> u & 1);
#pragma unroll
            for (int k = 0; k < VEC; ++k) {
                float keep = 1.f, write = 0.f;
                if (in) gates<T>(seq_to_float(rg[u].v[k]), keep, write);
                if (!BWD) {
                    B[u][k] = in ? write * seq_to_float(rx[u].v[k]) : 0.f;
                } else {
                    float before = 0.f;
                    if (in && !cut) before = t > 0 ? seq_to_float(rh[u].v[k]) : a.h_init ? a.h_init[c + k] : 0.f;
                    B[u][k] = in ? seq_to_float(rd[u].v[k]) : 0.f;
                    wr[u][k] = write;
                    df[u][k] = in ? (before - seq_to_float(rx[u].v[k])) * keep * write : 0.f;
                }
                A[u][k] = keep;
                if (RESET && cut) {
                    ps[k] = make_float2(SEQ_CUT, BWD ? 0.f : B[u][k]);
                    if (!BWD) A[u][k] = SEQ_CUT;
                } else {
                    if (!RESET || ps[k].x >= 0.f) ps[k].x *= keep;
                    ps[k].y = BWD ? keep * (B[u][k] + ps[k].y) : fmaf(keep, ps[k].y, B[u][k]);
                }
            }
        }
    }
#pragma unroll
    for (int k = 0; k < VEC; ++k) spans[sub][lane * VEC + k] = ps[k];
    __syncthreads();
    float2 before[VEC];  // the chunk's spans before this one
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
        float2 v[SUBS];
#pragma unroll
        for (int q = 0; q < SUBS; ++q) v[q] = spans[q][lane * VEC + k];
        float2 all = v[0];
        before[k] = make_float2(1.f, 0.f);
#pragma unroll
        for (int q = 1; q < SUBS; ++q) {
            if (q == sub) before[k] = all;
            all = join(all, v[q]);
        }
        if (sub == 0) whole[lane * VEC + k] = all;
    }
    __syncthreads();
    // the state entering the chunk, PER_WARP channels a warp
    {
        const int group = chunk >> 5, in_group = chunk & 31, section = group >> 5, in_section = group & 31;
        const int ch0 = sub * PER_WARP;
        unsigned long long *cp = DEEP ? wk.chunk_ps + (((long long)tile * wk.groups + group) * W + ch0) * 32 : nullptr;
        unsigned long long *gp = DEEP ? wk.group_ps + (((long long)tile * wk.sections + section) * W + ch0) * 32 : nullptr;
        unsigned long long *sp = DEEP ? wk.section + ((long long)tile * wk.sections + section) * W + ch0 : nullptr;
        const bool more = chunk + 1 < wk.chunks;
        if (DEEP && more && lane < PER_WARP) publish(cp + lane * 32 + in_group, whole[ch0 + lane]);
        if (DEEP && wk.test_wait && ticket == 0 && sub == 0) {
            unsigned left = wk.test_wait;
            while (!is_set(peek(sp)) && left-- > 0) {}  // (nothing enters the first section)
            if (lane == 0) seq_record(a.status + 1, WM_ERR_TIMEOUT);
        }
        // the group's chunks before this one; the group's (P, S) goes out before anything else is waited for
        float2 near[PER_WARP];
        if (DEEP && in_group) {
            unsigned long long p[PER_WARP];
#pragma unroll
            for (int q = 0; q < PER_WARP; ++q) p[q] = lane < in_group ? peek(cp + q * 32 + lane) : 0;
#pragma unroll
            for (int q = 0; q < PER_WARP; ++q) {
                near[q] = join_lanes(wait_for(p[q], cp + q * 32 + lane, lane < in_group, a.status));
                if (in_group == 31 && more && lane == 0) publish(gp + q * 32 + in_section, join(near[q], whole[ch0 + q]));
            }
        }
#pragma unroll
        for (int q = 0; q < PER_WARP; ++q) {
            const int ch = ch0 + q;
            float st = 0.f;
            if (!DEEP || section == 0) {
                if (j0 + ch < a.H && a.h0) st = a.h0[(long long)n * a.H + j0 + ch];
            } else {
                st = wait_for(peek(sp + q), sp + q, true, a.status).y;
            }
            if (DEEP && in_section) {
                const unsigned long long *p = gp + q * 32 + lane;
                st = through(join_lanes(wait_for(lane < in_section ? peek(p) : 0, p, lane < in_section, a.status)), st);
            }
            if (DEEP && in_group) st = through(near[q], st);
            if (lane == 0) {
                enter[ch] = st;
                st = through(whole[ch], st);
                if (DEEP && more && (chunk & 1023) == 1023) publish(sp + W + q, make_float2(0.f, st));
                if (!more && a.last && j0 + ch < a.H) a.last[(long long)n * a.H + j0 + ch] = st;
            }
        }
    }
    __syncthreads();
    // the outputs, from the state entering the span
    float mid[VEC];
#pragma unroll
    for (int k = 0; k < VEC; ++k) mid[k] = sub ? through(before[k], enter[lane * VEC + k]) : enter[lane * VEC + k];
    T *o0 = (BWD ? a.dgate.row(t0, n) : a.h.row(t0, n)) + j, *o1 = BWD ? a.dx.row(t0, n) + j : nullptr;
#pragma unroll
    for (int u = 0; u < L; ++u) {
        const long long t = BWD ? t0 - u : t0 + u;
        const bool in = t < live, cut = RESET && (cuts >> u & 1);
        V out0, out1;
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
            if (!BWD) {
                mid[k] = RESET && A[u][k] < 0.f ? B[u][k] : fmaf(A[u][k], mid[k], B[u][k]);
                out0.v[k] = seq_from_float<T>(in ? mid[k] : 0.f);
            } else {
                const float dL = B[u][k] + mid[k];
                out0.v[k] = seq_from_float<T>(in ? dL * df[u][k] : 0.f);
                out1.v[k] = seq_from_float<T>(in ? dL * wr[u][k] : 0.f);
                mid[k] = cut ? 0.f : A[u][k] * dL;
            }
        }
        if (mine && t >= 0 && t < T_) {
            seq_store(o0, out0);
            if (BWD) seq_store(o1, out1);
        }
        o0 += dir * (BWD ? a.dgate.st : a.h.st);
        if (BWD) o1 -= a.dx.st;
    }
}

__global__ void k_scan_state(long long C, const float *h0, float *last) {
    const long long c = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    if (c < C) last[c] = h0 ? h0[c] : 0.f;
}

// The largest of these numbers of values per access that alignment, strides and H allow.
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

template <class T, int VEC, bool BWD, bool RESET, int GROUPS>
cudaError_t stream_launch(const ScanParams<T> &q, size_t smem, cudaStream_t s) {
    auto *k = k_scan_stream<T, VEC, BWD, RESET, GROUPS>;
    cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    k<<<blocks(q.groups), kThreads, smem, s>>>(q);
    return cudaGetLastError();
}

// The deepest ring with which all CTAs run at once; 6 steps when there are more CTAs than that.
template <class T, int VEC, bool BWD>
cudaError_t stream(const wm_seq *h, const seq_scan_args &a, cudaStream_t s) {
    const ScanParams<T> q = params<T>(h, a, VEC, BWD);
    const size_t step = (BWD ? 4 : 2) * VEC * sizeof(T) * kThreads;
    const int per_sm = (int)((blocks(q.groups) + h->sms - 1) / h->sms);
    const size_t room = (size_t)(220 << 10) / per_sm;
    auto go = [&](auto reset) {
        constexpr bool R = decltype(reset)::value;
        if (room >= 12 * kGroup * step + 1024) return stream_launch<T, VEC, BWD, R, 12>(q, 12 * kGroup * step, s);
        if (room >= 6 * kGroup * step + 1024) return stream_launch<T, VEC, BWD, R, 6>(q, 6 * kGroup * step, s);
        return stream_launch<T, VEC, BWD, R, 3>(q, 3 * kGroup * step, s);
    };
    return a.reset ? go(std::true_type{}) : go(std::false_type{});
}

// What a call does: its kernel, the values per access, the steps per span and the layout of the
// workspace.
struct Plan {
    enum Kind { WALK, STREAM, SPANS } kind;
    int vec, len;
    SpanWork wk;  // offsets in bytes
    size_t ws;
};

Plan plan(const wm_seq *h, const seq_scan_args &a, bool bwd) {
    Plan p{};
    const int w4 = a.dtype == WM_BF16 ? 2 : 1;  // values in 4 bytes
    p.vec = width(a, bwd, 2 * w4);
    const long long C = (long long)a.N * a.H;
    if (a.T <= kWalk) {
        p.kind = Plan::WALK;
    } else if (p.vec >= w4 && C >= (long long)h->sms * 300) {
        p.kind = Plan::STREAM;
    } else {
        p.kind = Plan::SPANS;
        if (p.vec > w4) p.vec = w4;
        const int W = 32 * p.vec;
        SpanWork &k = p.wk;
        k.tiles_per_n = (a.H + W - 1) / W;
        k.tiles = a.N * k.tiles_per_n;
        // spans of 16 values a thread (backward 8); of 4 when the longer ones leave SMs idle
        p.len = (bwd ? 8 : 16);
        if ((a.T + SUBS * p.len - 1) / (SUBS * p.len) * k.tiles < h->sms) p.len = 4;
        k.chunks = (int)((a.T + SUBS * p.len - 1) / (SUBS * p.len));
        k.groups = (k.chunks + 31) / 32;
        k.sections = (k.groups + 31) / 32;
        if (k.chunks > 1) {
            const size_t t = (size_t)k.tiles * W * 8;
            p.ws = 256 + t * k.groups * 32 + t * k.sections * 32 + t * k.sections;
        }
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
        wk.group_ps = wk.chunk_ps + t * wk.groups * 32;
        wk.section = wk.group_ps + t * wk.sections * 32;
        wk.test_wait = h->test_wait;
        h->test_wait = 0;
        const cudaError_t e = cudaMemsetAsync(h->ws, 0xff, p.ws, s);
        if (e != cudaSuccess) return e;
        ++h->last_launches;
    }
    auto *k = a.reset ? (deep ? k_scan_spans<T, VEC, L, BWD, true, true> : k_scan_spans<T, VEC, L, BWD, true, false>)
                      : (deep ? k_scan_spans<T, VEC, L, BWD, false, true> : k_scan_spans<T, VEC, L, BWD, false, false>);
    k<<<(unsigned)((long long)wk.tiles * wk.chunks), kSpanThreads, 0, s>>>(q, wk);
    return cudaGetLastError();
}

template <class T, bool BWD>
cudaError_t dispatch(wm_seq *h, const seq_scan_args &a, cudaStream_t s) {
    constexpr int W4 = 4 / sizeof(T), LONG = BWD ? 8 : 16;
    const Plan p = plan(h, a, BWD);
    if (p.kind == Plan::WALK)
        return p.vec == 2 * W4 ? walk<T, 2 * W4, BWD>(h, a, s) : p.vec == W4 ? walk<T, W4, BWD>(h, a, s) : walk<T, 1, BWD>(h, a, s);
    if (p.kind == Plan::STREAM) return p.vec == 2 * W4 ? stream<T, 2 * W4, BWD>(h, a, s) : stream<T, W4, BWD>(h, a, s);
    if (p.vec == W4) return p.len == 4 ? spans<T, W4, 4, BWD>(h, a, p, s) : spans<T, W4, LONG, BWD>(h, a, p, s);
    return p.len == 4 ? spans<T, 1, 4, BWD>(h, a, p, s) : spans<T, 1, LONG, BWD>(h, a, p, s);
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
