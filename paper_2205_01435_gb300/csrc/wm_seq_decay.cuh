// wm_seq_decay.cuh -- what the kernels of the decayed linear attention share (see wm_seq_decay.cu).
// Not part of the public interface.
#pragma once
#include <cuda.h>

#include "wm_seq_internal.h"

// One array [T, N, H, D] of a call, strides in elements.
struct decay_array {
    const void *p;
    long long t, n, h;
};

// One pass over the sequences, in the order of time or against it: with X the state as the first token of a step sees it,
//   y_r = w_scale sum over j <= r of lambda^(r-j) (a_r . b_j) c_j + in_scale lambda^r X^T a_r
//   X' = lambda^n X + up_scale sum over j of lambda^(n-j) b_j c_j^T          after n tokens
// where sums do not reach past a cut (a reset, as seen from the side the pass comes from).
struct decay_job {
    decay_array a, b, c, y;
    int da, dc;              // values of a and b; of c and y
    int reverse;             // the tokens from the last to the first
    int first;               // the entering state has not decayed yet (time's order): X = lambda s_in; and it leaves so too
    int fine;                // the state is one that a call gives out: as good as in fp32 (whether it is asked for or not: outputs do not depend on that)
    int in_t, out_zero;      // s_in is [dc, da]; a reset of the token that comes last here empties s_out
    float w_scale, in_scale, up_scale;
    const float *s_in;       // [N, H, da, dc], or NULL = 0
    float *s_out;            // [N, H, da, dc], or NULL
    float *spans;            // split over time: [spans][N, H, da, dc], what a span's tokens give, then what enters it
    int spans_t;             // those are another job's: [dc, da], and that one forms them
    int vec;                 // values of a, b, c and y that one access may move (alignment)
    int map[3];              // which of q, k, v, dout a, b and c are
};

struct decay_pass {
    decay_job job[3];
    int jobs;
    long long T;
    int N, H;
    const float *log_decay;
    const uint8_t *reset;
    const int32_t *lengths;
    int *status;
    float *carry;            // [spans][2][N, H]: what a span multiplies the state by, by direction; < 0: it sees nothing before a cut
    int spans;               // of each sequence
    long long span_tokens;   // a multiple of the chunk
    int *redo;               // tensor-core pass: how many marks, then [jobs][N, H] marks: a chunk met what is not finite
    int only_redo;           // work on those alone
    uint32_t test_wait;      // > 0: the tensor-core pass's first CTA polls, that often, what nothing sets
};

// The tensor-core pass in bf16 (wm_seq_decay_tc.cu): its launch (state: only what the spans' tokens give the state), and the
// CTAs an SM holds.
constexpr int kDecayTcChunk = 128, kDecayTcMost = 128;  // tokens; values of a head
struct decay_maps {
    CUtensorMap in[4], out[3];  // of q, k, v, dout; of the jobs' outputs
    int use, stores;            // all inputs, all outputs have one
};
void wm_seq_decay_tc_maps(const seq_decay_args &a, const decay_pass &p, decay_maps &maps);
cudaError_t wm_seq_decay_tc_launch(wm_seq *h, const decay_pass &p, const decay_maps &maps, bool state, cudaStream_t s);
int wm_seq_decay_tc_ctas(int Dk, int Dv);

#ifdef __CUDACC__
// lambda^n: 1 for n = 0 whatever lambda is.
__device__ __forceinline__ float decay_power(float log_decay, long long n) { return n <= 0 ? 1.f : expf((float)n * log_decay); }

// Marks a job of a head of a sequence to be taken again.
__device__ __forceinline__ void decay_mark(const decay_pass &p, int job, long long pair) {
    if (atomicExch(p.redo + 1 + job * (long long)p.N * p.H + pair, 1) == 0) atomicAdd(p.redo, 1);
}

// A sequence as a pass sees it: step s of it is token at(s); steps from len on are padding.
struct decay_seq {
    long long T, len;
    int reverse;
    __device__ __forceinline__ long long at(long long s) const { return reverse && s < len ? len - 1 - s : s; }
};
__device__ __forceinline__ decay_seq decay_open(const decay_pass &p, const decay_job &j, int n) {
    long long len = p.T;
    if (p.lengths) {
        const int v = p.lengths[n];
        if (v < 0 || v > p.T) seq_record(p.status, WM_ERR_INVALID_ARG);
        len = max(0ll, min((long long)v, p.T));
    }
    return {p.T, len, j.reverse};
}
// A head that keeps nothing: each of its tokens begins something new (0 times a state that is not finite would be NaN).
__device__ __forceinline__ bool decay_keeps_none(float log_decay) { return log_decay == -INFINITY; }
// Does step s begin something new, seen in the pass's direction?
__device__ __forceinline__ bool decay_cut(const decay_pass &p, const decay_seq &q, long long s, int n, float log_decay) {
    if (s >= q.len) return false;
    if (decay_keeps_none(log_decay)) return !q.reverse || s > 0;
    if (!p.reset) return false;
    if (!q.reverse) return p.reset[s * p.N + n] != 0;
    return s > 0 && p.reset[(q.len - s) * p.N + n] != 0;  // (the token after this one, in time, begins an episode)
}
#endif
