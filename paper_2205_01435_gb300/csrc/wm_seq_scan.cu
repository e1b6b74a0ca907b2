// wm_seq_scan.cu -- the gated linear recurrence over time and its gradients.
//
//   keep = sigmoid(gate), write = 1 - keep;  h_t = keep_t h_{t-1} + write_t x_t
//   backward, from the last step down, with c the gradient flowing into h_t from later steps:
//   L = dh_t + c;  dx = L write;  dgate = L (h_{t-1} - x) keep write;  c = keep L
//
// A thread owns VEC neighbouring channels of one sequence and walks a span of steps with
// the state in fp32 registers.  Over a span the state is mapped by h -> P h + S, with P
// the product of its keeps and S its result from 0; a span that holds a reset ignores
// what enters it (P = SEQ_CUT).  When the channels alone do not fill the GPU, time is cut
// into spans: one launch forms each span's (P, S), one walks the spans of every channel
// and leaves the state entering each, and one runs all spans at once from there.
//
// Bound by memory: forward reads gate and x and writes h (6 bytes a value in bf16, about
// 8 operations), backward reads gate, x, h and dh and writes two gradients (12 bytes).
#include "wm_seq_internal.h"

namespace {

constexpr float SEQ_CUT = -1.f;  // P of a span with a reset inside (products of keeps are >= 0)
constexpr int kThreads = 128;

template <class T>
struct ScanParams {
    long long T_;
    int N, H, groups;  // groups: N * H / VEC
    int gpr;           // groups per sequence: H / VEC
    long long span;    // steps of a span
    int spans;
    seq_view<const T> gate, x, h_in, dh;
    seq_view<T> h, dgate, dx;
    const float *h0;      // what enters the first span, [N, H] (backward: dh_last), or null
    const float *h_init;  // backward: the forward's h0
    const uint8_t *reset;
    const int32_t *lengths;
    float *last;    // what leaves the last span, [N, H] (backward: dh0), or null
    float *sum_p, *sum_s;  // [spans, N * H]
    float *enter;          // [spans, N * H]
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

// One span of one thread's channels from the state in st (backward: the gradient).  OUT: write
// the outputs; else only the state is carried, and P is the product of the keeps.
template <class T, int VEC, bool BWD, bool OUT>
__device__ __forceinline__ void walk(const ScanParams<T> &a, int n, int j, long long t_lo, long long t_hi, float (&st)[VEC],
                                     float (&P)[VEC]) {
    constexpr int U = VEC * sizeof(T) >= 16 ? 4 : 8;  // steps whose loads are in flight together
    using V = seq_vec<T, VEC>;
    const T *g = a.gate.p + n * a.gate.sn + j;
    const T *x = (BWD && !OUT) ? nullptr : a.x.p + n * a.x.sn + j;
    const T *dh = BWD ? a.dh.p + n * a.dh.sn + j : nullptr;
    const T *hp = BWD && OUT ? a.h_in.p + n * a.h_in.sn + j : nullptr;
    const uint8_t *rs = a.reset ? a.reset + n : nullptr;
    for (long long i = t_lo; i < t_hi; i += U) {
        V vg[U], vx[U], vd[U], vh[U];
        uint8_t vr[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            // forward i, i + 1, ...; backward the mirrored steps
            const long long t = BWD ? t_lo + (t_hi - 1 - (i + u)) : i + u;
            if (i + u < t_hi) {
                vg[u] = seq_load<T, VEC>(g + t * a.gate.st);
                if (!BWD || OUT) vx[u] = seq_load<T, VEC>(x + t * a.x.st);
                if (BWD) vd[u] = seq_load<T, VEC>(dh + t * a.dh.st);
                if (BWD && OUT && t > 0) vh[u] = seq_load<T, VEC>(hp + (t - 1) * a.h_in.st);
                vr[u] = rs ? rs[t * a.N] : 0;
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (i + u >= t_hi) break;
            const long long t = BWD ? t_lo + (t_hi - 1 - (i + u)) : i + u;
            const bool cut = vr[u] != 0;
            V o0, o1;
#pragma unroll
            for (int k = 0; k < VEC; ++k) {
                float keep, write;
                gates<T>(seq_to_float(vg[u].v[k]), keep, write);
                if (!BWD) {
                    const float before = cut ? 0.f : st[k];
                    st[k] = fmaf(keep, before, write * seq_to_float(vx[u].v[k]));
                    if (OUT) o0.v[k] = seq_from_float<T>(st[k]);
                } else {
                    const float L = seq_to_float(vd[u].v[k]) + st[k];
                    if (OUT) {
                        float before = 0.f;
                        if (!cut) before = t > 0 ? seq_to_float(vh[u].v[k])
                                                 : a.h_init ? a.h_init[(long long)n * a.H + j + k] : 0.f;
                        o0.v[k] = seq_from_float<T>(L * (before - seq_to_float(vx[u].v[k])) * keep * write);
                        o1.v[k] = seq_from_float<T>(L * write);
                    }
                    st[k] = cut ? 0.f : keep * L;
                }
                if (!OUT) P[k] = cut || P[k] < 0.f ? SEQ_CUT : P[k] * keep;
            }
            if (OUT) {
                if (!BWD) {
                    seq_store(a.h.p + t * a.h.st + n * a.h.sn + j, o0);
                } else {
                    seq_store(a.dgate.p + t * a.dgate.st + n * a.dgate.sn + j, o0);
                    seq_store(a.dx.p + t * a.dx.st + n * a.dx.sn + j, o1);
                }
            }
        }
    }
}

// SUM: the spans' (P, S).  Else the outputs, from `enter` (or h0, when there is one span).
template <class T, int VEC, bool BWD, bool SUM>
__global__ void __launch_bounds__(kThreads) k_seq_scan(const ScanParams<T> a) {
    const int grp = blockIdx.x * kThreads + threadIdx.x;
    if (grp >= a.groups) return;
    const int n = grp / a.gpr, j = (grp - n * a.gpr) * VEC;
    const long long c = (long long)n * a.H + j, C = (long long)a.N * a.H;
    const int sp = blockIdx.y;
    const long long live = live_steps(a.lengths, n, a.T_, a.status);
    const long long t0 = sp * a.span, t1 = min(a.T_, t0 + a.span);
    const long long mid = max(t0, min(t1, live));  // steps [mid, t1) are padding
    float st[VEC], P[VEC];
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
        P[k] = 1.f;
        st[k] = SUM ? 0.f : a.spans > 1 ? a.enter[sp * C + c + k] : a.h0 ? a.h0[c + k] : 0.f;
    }
    walk<T, VEC, BWD, !SUM>(a, n, j, t0, mid, st, P);
    if (SUM) {
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
            a.sum_p[sp * C + c + k] = P[k];
            a.sum_s[sp * C + c + k] = st[k];
        }
        return;
    }
    seq_vec<T, VEC> zero;
#pragma unroll
    for (int k = 0; k < VEC; ++k) zero.v[k] = seq_from_float<T>(0.f);
    for (long long t = mid; t < t1; ++t) {
        if (!BWD) {
            seq_store(a.h.p + t * a.h.st + n * a.h.sn + j, zero);
        } else {
            seq_store(a.dgate.p + t * a.dgate.st + n * a.dgate.sn + j, zero);
            seq_store(a.dx.p + t * a.dx.st + n * a.dx.sn + j, zero);
        }
    }
    if (a.last && a.spans == 1) {
#pragma unroll
        for (int k = 0; k < VEC; ++k) a.last[c + k] = st[k];
    }
}

// The state entering every span of a channel, and what leaves the last.
template <bool BWD>
__global__ void __launch_bounds__(kThreads) k_seq_join(int spans, long long C, const float *__restrict__ h0,
                                                       const float *__restrict__ sum_p, const float *__restrict__ sum_s,
                                                       float *__restrict__ enter, float *last) {
    const long long c = (long long)blockIdx.x * kThreads + threadIdx.x;
    if (c >= C) return;
    float st = h0 ? h0[c] : 0.f;
    for (int i = 0; i < spans; ++i) {
        const int sp = BWD ? spans - 1 - i : i;
        const float p = sum_p[sp * C + c], s = sum_s[sp * C + c];
        enter[sp * C + c] = st;
        st = p < 0.f ? s : fmaf(p, st, s);
    }
    if (last) last[c] = st;
}

__global__ void k_seq_state(long long C, const float *h0, float *last) {
    const long long c = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    if (c < C) last[c] = h0 ? h0[c] : 0.f;
}

struct Plan {
    int vec, spans;
    long long span;
};

bool divides(const wm_seq_view &v, int vec, size_t es) {
    return (uintptr_t)v.data % (vec * es) == 0 && v.stride_t % vec == 0 && v.stride_n % vec == 0;
}

Plan plan(const wm_seq *h, const seq_scan_args &a, bool bwd) {
    const size_t es = a.dtype == WM_BF16 ? 2 : 4;
    int vec = 16 / (int)es;
    auto fits = [&](int v) {
        return a.H % v == 0 && divides(a.gate, v, es) && divides(a.x, v, es) && divides(a.h, v, es) &&
               (!bwd || (divides(a.dh, v, es) && divides(a.dgate, v, es) && divides(a.dx, v, es)));
    };
    while (vec > 1 && !fits(vec)) vec /= 2;
    Plan p{vec, 1, a.T > 0 ? a.T : 1};
    // enough threads for every SM's loads in flight
    const long long groups = (long long)a.N * a.H / vec, want = (long long)h->sms * 512;
    if (groups < want / 2 && a.T >= 64) {
        long long spans = (want + groups - 1) / groups;
        if (spans > a.T / 32) spans = a.T / 32;
        p.span = (a.T + spans - 1) / spans;
        p.spans = (int)((a.T + p.span - 1) / p.span);
    }
    return p;
}

template <class T>
ScanParams<T> params(const wm_seq *h, const seq_scan_args &a, const Plan &p, bool bwd) {
    ScanParams<T> q{};
    q.T_ = a.T; q.N = a.N; q.H = a.H;
    q.gpr = a.H / p.vec; q.groups = a.N * q.gpr;
    q.span = p.span; q.spans = p.spans;
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
    const size_t n = (size_t)p.spans * a.N * a.H;
    q.sum_p = (float *)h->ws; q.sum_s = q.sum_p + n; q.enter = q.sum_s + n;
    return q;
}

template <class T, int VEC, bool BWD>
void launch(wm_seq *h, const ScanParams<T> &q, cudaStream_t s) {
    const dim3 grid((q.groups + kThreads - 1) / kThreads, q.spans);
    if (q.spans > 1) {
        const long long C = (long long)q.N * q.H;
        k_seq_scan<T, VEC, BWD, true><<<grid, kThreads, 0, s>>>(q);
        k_seq_join<BWD><<<(unsigned)((C + kThreads - 1) / kThreads), kThreads, 0, s>>>(q.spans, C, q.h0, q.sum_p, q.sum_s,
                                                                                       q.enter, q.last);
        h->last_launches = 2;
    }
    k_seq_scan<T, VEC, BWD, false><<<grid, kThreads, 0, s>>>(q);
    ++h->last_launches;
}

template <class T, bool BWD>
void dispatch(wm_seq *h, const seq_scan_args &a, const Plan &p, cudaStream_t s) {
    const ScanParams<T> q = params<T>(h, a, p, BWD);
    if constexpr (sizeof(T) == 2)
        if (p.vec == 8) return launch<T, 8, BWD>(h, q, s);
    if (p.vec == 4) return launch<T, 4, BWD>(h, q, s);
    if (p.vec == 2) return launch<T, 2, BWD>(h, q, s);
    launch<T, 1, BWD>(h, q, s);
}

}  // namespace

size_t wm_seq_scan_ws(const wm_seq *h, const seq_scan_args &a, bool backward) {
    const Plan p = plan(h, a, backward);
    return p.spans > 1 ? (size_t)p.spans * a.N * a.H * 3 * sizeof(float) : 0;
}

cudaError_t wm_seq_scan_launch(wm_seq *h, const seq_scan_args &a, bool backward, cudaStream_t s) {
    h->last_launches = 0;
    if (a.T == 0) {  // the state goes through
        float *last = backward ? a.dh0 : a.h_last;
        if (last) {
            const long long C = (long long)a.N * a.H;
            k_seq_state<<<(unsigned)((C + 255) / 256), 256, 0, s>>>(C, backward ? a.dh_last : a.h0, last);
            h->last_launches = 1;
        }
        return cudaGetLastError();
    }
    const Plan p = plan(h, a, backward);
    if (a.dtype == WM_BF16)
        backward ? dispatch<__nv_bfloat16, true>(h, a, p, s) : dispatch<__nv_bfloat16, false>(h, a, p, s);
    else
        backward ? dispatch<float, true>(h, a, p, s) : dispatch<float, false>(h, a, p, s);
    return cudaGetLastError();
}
