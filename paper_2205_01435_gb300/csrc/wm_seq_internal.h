// wm_seq_internal.h -- handle, checks and launchers behind the C ABI of include/wm_seq.h.
// Not part of the public interface.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <mutex>

#include "wm_seq.h"

struct wm_seq {
    std::mutex busy;  // held by a call: the binding gives up the interpreter's lock, which kept threads apart
    int device = 0;
    int sms = 0;
    int sort_ranks = 0;  // CTAs of the embedding gradient's sorting cluster, at most
    int clip_ctas = 0;   // CTAs of the one-launch clipping, at most
    void *ws = nullptr;  // workspace (grows on demand)
    size_t ws_bytes = 0;
    bool ws_captured = false;   // a captured graph may hold ws: it is kept when ws grows
    void *retired[64] = {};     // such earlier workspaces (each at least doubles)
    int n_retired = 0;
    // 64 device words: [0] status: arguments, [1] status: a wait gave up; [8] and [16, 17] counters
    // that the clipping's CTAs meet at (0 between calls)
    int *status = nullptr;
    int last_launches = 0;
    uint32_t test_wait = 0;     // wm_seq_inject_wait_timeout: polls of the next call's injected wait
    char err[256] = "";
};

// A [T, N, H] view on the device (strides in elements).
template <class P>
struct seq_view {
    P *p;
    long long st, sn;
    __device__ __forceinline__ P *row(long long t, long long n) const { return p + t * st + n * sn; }
};

struct seq_scan_args {
    int dtype;
    long long T;
    int N, H;
    wm_seq_view gate, x, h, dh, dgate, dx;  // forward: gate, x in, h out; backward: h in
    const float *h0, *dh_last;
    const uint8_t *reset;
    const int32_t *lengths;
    float *h_last, *dh0;
};

// What the launchers ask the device for, once a handle.
cudaError_t wm_seq_embed_prepare(wm_seq *h);
cudaError_t wm_seq_clip_prepare(wm_seq *h);

// ---- launchers.  *_ws: bytes of workspace a call takes ------------------------------
size_t wm_seq_scan_ws(const wm_seq *h, const seq_scan_args &a, bool backward);
cudaError_t wm_seq_scan_launch(wm_seq *h, const seq_scan_args &a, bool backward, cudaStream_t s);

cudaError_t wm_seq_norm_launch(wm_seq *h, int dtype, long long rows, int D, const void *x, long long ldx,
                               const float *w, const float *b, float eps, void *y, long long ldy, float *mean,
                               float *rstd, cudaStream_t s);
size_t wm_seq_norm_backward_ws(const wm_seq *h, int dtype, long long rows, int D, const void *x, long long ldx, const void *dy,
                               long long lddy, const void *dx, long long lddx);
cudaError_t wm_seq_norm_backward_launch(wm_seq *h, int dtype, long long rows, int D, const void *x, long long ldx,
                                        const float *w, const float *mean, const float *rstd, const void *dy,
                                        long long lddy, void *dx, long long lddx, float *dw, float *db,
                                        cudaStream_t s);

cudaError_t wm_seq_embed_launch(wm_seq *h, int dtype, long long n, int V, int D, const void *table,
                                const int32_t *tokens, float scale, void *out, cudaStream_t s);
size_t wm_seq_embed_backward_ws(const wm_seq *h, int dtype, long long n, int V, int D, const void *dout, const void *dtable);
cudaError_t wm_seq_embed_backward_launch(wm_seq *h, int dtype, long long n, int V, int D, const int32_t *tokens,
                                         const void *dout, float scale, void *dtable, cudaStream_t s);

size_t wm_seq_clip_ws(const wm_seq *h);
cudaError_t wm_seq_clip_launch(wm_seq *h, int count, const wm_seq_grad *grads, float max_norm, float *norm,
                               cudaStream_t s);

// ---- device helpers -----------------------------------------------------------------
#ifdef __CUDACC__
// Records the first error; later ones keep it.
__device__ __forceinline__ void seq_record(int *status, int code) { atomicCAS(status, 0, code); }

__device__ __forceinline__ float seq_to_float(float v) { return v; }
__device__ __forceinline__ float seq_to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
template <class T>
__device__ __forceinline__ T seq_from_float(float v);
template <>
__device__ __forceinline__ float seq_from_float<float>(float v) {
    return v;
}
template <>
__device__ __forceinline__ __nv_bfloat16 seq_from_float<__nv_bfloat16>(float v) {
    return __float2bfloat16_rn(v);
}

// VEC values of type T that one access moves (at most 16 bytes); aligned to their size.
template <class T, int VEC>
struct alignas(sizeof(T) * VEC) seq_vec {
    T v[VEC];
};
template <class T, int VEC>
__device__ __forceinline__ seq_vec<T, VEC> seq_load(const T *p) {
    return *reinterpret_cast<const seq_vec<T, VEC> *>(p);
}
// The values of a vector as floats, and back; bf16 in pairs (one instruction a value, or two values).
template <class T, int VEC>
__device__ __forceinline__ void seq_unpack(const seq_vec<T, VEC> &v, float (&f)[VEC]) {
    if constexpr (sizeof(T) == 2 && VEC % 2 == 0) {
        const uint32_t *w = reinterpret_cast<const uint32_t *>(&v);
#pragma unroll
        for (int k = 0; k < VEC / 2; ++k) {
            f[2 * k] = __uint_as_float(w[k] << 16);
            f[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int k = 0; k < VEC; ++k) f[k] = seq_to_float(v.v[k]);
    }
}
template <class T, int VEC>
__device__ __forceinline__ seq_vec<T, VEC> seq_pack(const float (&f)[VEC]) {
    seq_vec<T, VEC> v;
    if constexpr (sizeof(T) == 2 && VEC % 2 == 0) {
        __nv_bfloat162 *w = reinterpret_cast<__nv_bfloat162 *>(&v);
#pragma unroll
        for (int k = 0; k < VEC / 2; ++k) w[k] = __floats2bfloat162_rn(f[2 * k], f[2 * k + 1]);
    } else {
#pragma unroll
        for (int k = 0; k < VEC; ++k) v.v[k] = seq_from_float<T>(f[k]);
    }
    return v;
}
template <class T, int VEC>
__device__ __forceinline__ void seq_store(T *p, const seq_vec<T, VEC> &v) {
    *reinterpret_cast<seq_vec<T, VEC> *>(p) = v;
}

// ---- asynchronous copies into a thread's own places of shared memory (4, 8 or 16 bytes) ----
template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t dst, const void *src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
#endif
