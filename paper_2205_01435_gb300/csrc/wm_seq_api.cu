// wm_seq_api.cu -- the C ABI of include/wm_seq.h: argument checks, the handle and its
// workspace, and the calls of the operators' launchers.
#include <math.h>
#include <stdio.h>

#include <new>

#include "wm_seq_internal.h"

namespace {

wm_status fail(wm_seq *h, wm_status st, const char *what, const char *why) {
    if (h) snprintf(h->err, sizeof h->err, "%s: %s", what, why);
    return st;
}

// (The runtime keeps a failing call's error until it is asked for: the next launch would report it again.)
wm_status cuda_fail(wm_seq *h, cudaError_t e, const char *what) {
    cudaGetLastError();
    return fail(h, e == cudaErrorMemoryAllocation ? WM_ERR_OOM : WM_ERR_CUDA, what, cudaGetErrorString(e));
}

// Makes the handle's device current for the scope of a call.
struct OnDevice {
    int before = 0;
    bool changed = false;
    cudaError_t e;
    explicit OnDevice(const wm_seq *h) {
        e = cudaGetDevice(&before);
        if (e == cudaSuccess && before != h->device) {
            e = cudaSetDevice(h->device);
            changed = e == cudaSuccess;
        }
    }
    ~OnDevice() {
        if (changed) cudaSetDevice(before);
    }
};

// Collects the checks of a call's arguments: the first that fails stays.
struct Check {
    const wm_seq *h;
    const char *why = nullptr;
    void that(bool ok, const char *msg) {
        if (!ok && !why) why = msg;
    }
    // an array of the device (aligned to its elements); `needed`: NULL is an error
    void array(const void *p, size_t align, bool needed, const char *msg) {
        if (why) return;
        if (!p) {
            that(!needed, msg);
            return;
        }
        if ((uintptr_t)p % align) {
            that(false, "an array is not aligned to its element size");
            return;
        }
        cudaPointerAttributes at;
        if (cudaPointerGetAttributes(&at, p) != cudaSuccess) {
            cudaGetLastError();
            that(false, "an array's address is not known to CUDA");
            return;
        }
        const bool here = at.type == cudaMemoryTypeManaged ||
                          (at.type == cudaMemoryTypeDevice && at.device == h->device);
        that(here, "arrays must be memory of the handle's device (host arrays are not staged)");
    }
    void view(const wm_seq_view *v, long long T, int N, int H, size_t esize, bool out, bool needed, const char *msg) {
        if (why) return;
        if (!v) {
            that(!needed, msg);
            return;
        }
        array(v->data, esize, needed, msg);
        that(v->stride_t >= 0 && v->stride_n >= 0, "strides must be >= 0");
        if (why || !out) return;
        // apart: one axis steps over the whole extent of the other
        const __int128 st = v->stride_t, sn = v->stride_n;  // (products pass 64 bits for absurd strides)
        const bool t_outer = (T <= 1 || st >= (N - 1) * sn + H) && (N <= 1 || sn >= H);
        const bool n_outer = (N <= 1 || sn >= (T - 1) * st + H) && (T <= 1 || st >= H);
        that(t_outer || n_outer, "an output's elements overlap (strides)");
    }
};

size_t esize(int dtype) { return dtype == WM_BF16 ? 2 : 4; }

// The longest rows, and the most tokens: the kernels' 32-bit indices go past the end by less than 65,536.
constexpr long long kMostInt = (1ll << 31) - 65536;

// Room for `need` bytes of scratch on the handle, for a call on stream s.
wm_status reserve(wm_seq *h, size_t need, cudaStream_t s, const char *what) {
    if (need == 0) return WM_OK;
    cudaStreamCaptureStatus cs = cudaStreamCaptureStatusNone;
    cudaError_t e = cudaStreamIsCapturing(s, &cs);
    if (e != cudaSuccess) return cuda_fail(h, e, what);
    const bool capturing = cs != cudaStreamCaptureStatusNone;
    if (need > h->ws_bytes) {
        if (capturing)
            return fail(h, WM_ERR_UNSUPPORTED, what,
                        "the workspace would have to grow under stream capture: make a call of this size first");
        if (h->ws_captured && h->n_retired == 64)
            return fail(h, WM_ERR_OOM, what, "too many captured graphs hold earlier workspaces of this handle");
        size_t n = need + need / 8;
        if (n < 2 * h->ws_bytes) n = 2 * h->ws_bytes;
        if ((e = cudaDeviceSynchronize()) != cudaSuccess) return cuda_fail(h, e, what);
        void *p = nullptr;
        e = cudaMalloc(&p, n);
        if (e != cudaSuccess) {
            cudaGetLastError();
            if ((e = cudaMalloc(&p, n = need)) != cudaSuccess) return cuda_fail(h, e, what);
        }
        if (h->ws) {
            if (h->ws_captured)
                h->retired[h->n_retired++] = h->ws;
            else
                cudaFree(h->ws);
        }
        h->ws = p;
        h->ws_bytes = n;
        h->ws_captured = false;
    }
    if (capturing) h->ws_captured = true;
    return WM_OK;
}

// Clears the first `bytes` of the status words, and waits for it: a memset of device memory returns before it
// has run, and nothing orders it before the caller's next launch on a stream that does not wait for the default one.
cudaError_t clear_status(wm_seq *h, size_t bytes) {
    const cudaError_t e = cudaMemset(h->status, 0, bytes);
    return e == cudaSuccess ? cudaStreamSynchronize(cudaStreamLegacy) : e;
}

wm_status launched(wm_seq *h, cudaError_t e, const char *what) {
    return e == cudaSuccess ? WM_OK : cuda_fail(h, e, what);
}

}  // namespace

extern "C" wm_status wm_seq_create(wm_seq **out) {
    if (!out) return WM_ERR_INVALID_ARG;
    *out = nullptr;
    wm_seq *h = new (std::nothrow) wm_seq;
    if (!h) return WM_ERR_OOM;
    cudaError_t e = cudaGetDevice(&h->device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&h->sms, cudaDevAttrMultiProcessorCount, h->device);
    if (e == cudaSuccess) e = cudaMalloc((void **)&h->status, 256);
    if (e == cudaSuccess) e = clear_status(h, 256);
    if (e == cudaSuccess) e = wm_seq_embed_prepare(h);
    if (e == cudaSuccess) e = wm_seq_clip_prepare(h);
    if (e != cudaSuccess) {
        cudaGetLastError();
        if (h->status) cudaFree(h->status);
        delete h;
        return e == cudaErrorMemoryAllocation ? WM_ERR_OOM : WM_ERR_CUDA;
    }
    *out = h;
    return WM_OK;
}

extern "C" void wm_seq_destroy(wm_seq *h) {
    if (!h) return;
    {
        OnDevice on(h);
        cudaDeviceSynchronize();
        for (int i = 0; i < h->n_retired; ++i) cudaFree(h->retired[i]);
        if (h->ws) cudaFree(h->ws);
        if (h->status) cudaFree(h->status);
    }
    delete h;
}

extern "C" wm_status wm_seq_sync(wm_seq *h) {
    if (!h) return WM_ERR_INVALID_ARG;
    const std::lock_guard<std::mutex> busy(h->busy);
    h->err[0] = 0;
    OnDevice on(h);
    int st[2] = {};
    cudaError_t e = on.e;
    if (e == cudaSuccess) e = cudaDeviceSynchronize();
    if (e == cudaSuccess) e = cudaMemcpy(st, h->status, sizeof st, cudaMemcpyDeviceToHost);
    // (with a wait that gave up, the counters that calls meet at are reset too)
    if (e == cudaSuccess && (st[0] || st[1])) e = clear_status(h, st[1] ? 256 : sizeof st);
    if (e != cudaSuccess) return cuda_fail(h, e, "wm_seq_sync");
    if (st[1]) return fail(h, (wm_status)st[1], "wm_seq_sync", "a wait inside a kernel gave up");
    if (st[0]) return fail(h, (wm_status)st[0], "wm_seq_sync", "a token or a length of an earlier call was out of range");
    return WM_OK;
}

extern "C" const char *wm_seq_last_error(const wm_seq *h) { return h ? h->err : "null handle"; }

extern "C" int wm_seq_last_launches(const wm_seq *h) { return h ? h->last_launches : 0; }

extern "C" wm_status wm_seq_inject_wait_timeout(wm_seq *h, unsigned int polls) {
    if (!h) return WM_ERR_INVALID_ARG;
    const std::lock_guard<std::mutex> busy(h->busy);
    h->err[0] = 0;
    h->test_wait = polls;
    return WM_OK;
}

#define SEQ_BEGIN(what)                                            \
    if (!h) return WM_ERR_INVALID_ARG;                             \
    const std::lock_guard<std::mutex> busy(h->busy);               \
    h->err[0] = 0;                                                 \
    static const char *const kWhat = what;                         \
    OnDevice on(h);                                                \
    if (on.e != cudaSuccess) return cuda_fail(h, on.e, kWhat);     \
    Check c{h};                                                    \
    const cudaStream_t s = (cudaStream_t)cuda_stream;
#define SEQ_DTYPE() c.that(dtype == WM_FP32 || dtype == WM_BF16, "dtype must be WM_FP32 or WM_BF16")
#define SEQ_CHECKED() \
    if (c.why) return fail(h, WM_ERR_INVALID_ARG, kWhat, c.why)

extern "C" wm_status wm_seq_embed(wm_seq *h, int dtype, long long n, int V, int D, const void *table,
                                  const int32_t *tokens, float scale, void *out, void *cuda_stream) {
    SEQ_BEGIN("wm_seq_embed");
    SEQ_DTYPE();
    c.that(n >= 0 && V >= 1 && D >= 1 && D <= kMostInt, "n >= 0, V >= 1 and 1 <= D <= 2^31 - 65536 are needed");
    SEQ_CHECKED();
    c.array(table, esize(dtype), n > 0, "table is NULL");
    c.array(tokens, 4, n > 0, "tokens is NULL");
    c.array(out, esize(dtype), n > 0, "out is NULL");
    SEQ_CHECKED();
    h->last_launches = 0;
    if (n == 0) return WM_OK;
    return launched(h, wm_seq_embed_launch(h, dtype, n, V, D, table, tokens, scale, out, s), kWhat);
}

extern "C" wm_status wm_seq_embed_backward(wm_seq *h, int dtype, long long n, int V, int D, const int32_t *tokens,
                                           const void *dout, float scale, void *dtable, void *cuda_stream) {
    SEQ_BEGIN("wm_seq_embed_backward");
    SEQ_DTYPE();
    c.that(n >= 0 && n <= kMostInt && V >= 1 && D >= 1 && D <= kMostInt,
           "0 <= n <= 2^31 - 65536, V >= 1 and 1 <= D <= 2^31 - 65536 are needed");
    SEQ_CHECKED();
    c.array(tokens, 4, n > 0, "tokens is NULL");
    c.array(dout, esize(dtype), n > 0, "dout is NULL");
    c.array(dtable, esize(dtype), true, "dtable is NULL");
    SEQ_CHECKED();
    const wm_status st = reserve(h, wm_seq_embed_backward_ws(h, dtype, n, V, D, dout, dtable), s, kWhat);
    if (st != WM_OK) return st;
    return launched(h, wm_seq_embed_backward_launch(h, dtype, n, V, D, tokens, dout, scale, dtable, s), kWhat);
}

extern "C" wm_status wm_seq_layer_norm(wm_seq *h, int dtype, long long rows, int D, const void *x, long long ldx,
                                       const float *weight, const float *bias, float eps, void *y, long long ldy,
                                       float *mean, float *rstd, void *cuda_stream) {
    SEQ_BEGIN("wm_seq_layer_norm");
    SEQ_DTYPE();
    c.that(rows >= 0 && D >= 1 && D <= kMostInt, "rows >= 0 and 1 <= D <= 2^31 - 65536 are needed");
    c.that(eps >= 0.f && !isinf(eps), "eps must be finite and >= 0");
    c.that(ldx >= 0, "ldx must be >= 0");
    c.that(rows <= 1 || ldy >= D, "ldy must be >= D");
    c.that(!mean == !rstd, "mean and rstd are given together");
    SEQ_CHECKED();
    c.array(x, esize(dtype), rows > 0, "x is NULL");
    c.array(y, esize(dtype), rows > 0, "y is NULL");
    c.array(weight, 4, false, "");
    c.array(bias, 4, false, "");
    c.array(mean, 4, false, "");
    c.array(rstd, 4, false, "");
    c.that(x != y || ldx == ldy || rows <= 1, "y may be x with the same row stride only");
    SEQ_CHECKED();
    h->last_launches = 0;
    if (rows == 0) return WM_OK;
    return launched(h, wm_seq_norm_launch(h, dtype, rows, D, x, ldx, weight, bias, eps, y, ldy, mean, rstd, s), kWhat);
}

extern "C" wm_status wm_seq_layer_norm_backward(wm_seq *h, int dtype, long long rows, int D, const void *x,
                                                long long ldx, const float *weight, const float *mean,
                                                const float *rstd, const void *dy, long long lddy, void *dx,
                                                long long lddx, float *dweight, float *dbias, void *cuda_stream) {
    SEQ_BEGIN("wm_seq_layer_norm_backward");
    SEQ_DTYPE();
    c.that(rows >= 0 && D >= 1 && D <= kMostInt, "rows >= 0 and 1 <= D <= 2^31 - 65536 are needed");
    c.that(ldx >= 0 && lddy >= 0, "ldx and lddy must be >= 0");
    c.that(rows <= 1 || lddx >= D, "lddx must be >= D");
    SEQ_CHECKED();
    c.array(x, esize(dtype), rows > 0, "x is NULL");
    c.array(dy, esize(dtype), rows > 0, "dy is NULL");
    c.array(dx, esize(dtype), rows > 0, "dx is NULL");
    c.array(mean, 4, rows > 0, "mean is NULL");
    c.array(rstd, 4, rows > 0, "rstd is NULL");
    c.array(weight, 4, false, "");
    c.array(dweight, 4, false, "");
    c.array(dbias, 4, false, "");
    c.that(dx != dy || lddx == lddy || rows <= 1, "dx may be dy with the same row stride only");
    c.that(dx != x || rows == 0, "dx must not be x");
    SEQ_CHECKED();
    const wm_status st = reserve(h, wm_seq_norm_backward_ws(h, dtype, rows, D, x, ldx, dy, lddy, dx, lddx), s, kWhat);
    if (st != WM_OK) return st;
    return launched(h, wm_seq_norm_backward_launch(h, dtype, rows, D, x, ldx, weight, mean, rstd, dy, lddy, dx, lddx,
                                                   dweight, dbias, s), kWhat);
}

extern "C" wm_status wm_seq_gated_scan(wm_seq *h, int dtype, long long T, int N, int H, const wm_seq_view *gate,
                                       const wm_seq_view *x, const float *h0, const uint8_t *reset,
                                       const int32_t *lengths, const wm_seq_view *out, float *h_last,
                                       void *cuda_stream) {
    SEQ_BEGIN("wm_seq_gated_scan");
    SEQ_DTYPE();
    c.that(T >= 0 && T <= kMostInt && N >= 0 && H >= 1 && H <= kMostInt,
           "0 <= T <= 2^31 - 65536, N >= 0 and 1 <= H <= 2^31 - 65536 are needed");
    c.that((long long)N * ((H + 31ll) / 32) < (1ll << 31), "N * ceil(H / 32) must be below 2^31");
    SEQ_CHECKED();
    const bool any = T > 0 && N > 0;
    const size_t es = esize(dtype);
    c.view(gate, T, N, H, es, false, any, "gate is NULL");
    c.view(x, T, N, H, es, false, any, "x is NULL");
    c.view(out, T, N, H, es, true, any, "out is NULL");
    c.array(h0, 4, false, "");
    c.array(reset, 1, false, "");
    c.array(lengths, 4, false, "");
    c.array(h_last, 4, false, "");
    SEQ_CHECKED();
    h->last_launches = 0;
    if (N == 0) return WM_OK;
    seq_scan_args a{};
    a.dtype = dtype; a.T = T; a.N = N; a.H = H;
    if (any) {
        a.gate = *gate; a.x = *x; a.h = *out;
    }
    a.h0 = h0; a.reset = reset; a.lengths = lengths; a.h_last = h_last;
    const wm_status st = reserve(h, wm_seq_scan_ws(h, a, false), s, kWhat);
    if (st != WM_OK) return st;
    return launched(h, wm_seq_scan_launch(h, a, false, s), kWhat);
}

extern "C" wm_status wm_seq_gated_scan_backward(wm_seq *h, int dtype, long long T, int N, int H,
                                                const wm_seq_view *gate, const wm_seq_view *x, const float *h0,
                                                const uint8_t *reset, const int32_t *lengths,
                                                const wm_seq_view *h_seq, const wm_seq_view *dh, const float *dh_last,
                                                const wm_seq_view *dgate, const wm_seq_view *dx, float *dh0,
                                                void *cuda_stream) {
    SEQ_BEGIN("wm_seq_gated_scan_backward");
    SEQ_DTYPE();
    c.that(T >= 0 && T <= kMostInt && N >= 0 && H >= 1 && H <= kMostInt,
           "0 <= T <= 2^31 - 65536, N >= 0 and 1 <= H <= 2^31 - 65536 are needed");
    c.that((long long)N * ((H + 31ll) / 32) < (1ll << 31), "N * ceil(H / 32) must be below 2^31");
    SEQ_CHECKED();
    const bool any = T > 0 && N > 0;
    const size_t es = esize(dtype);
    c.view(gate, T, N, H, es, false, any, "gate is NULL");
    c.view(x, T, N, H, es, false, any, "x is NULL");
    c.view(h_seq, T, N, H, es, false, any, "h_seq is NULL");
    c.view(dh, T, N, H, es, false, any, "dh is NULL");
    c.view(dgate, T, N, H, es, true, any, "dgate is NULL");
    c.view(dx, T, N, H, es, true, any, "dx is NULL");
    c.array(h0, 4, false, "");
    c.array(reset, 1, false, "");
    c.array(lengths, 4, false, "");
    c.array(dh_last, 4, false, "");
    c.array(dh0, 4, false, "");
    SEQ_CHECKED();
    h->last_launches = 0;
    if (N == 0) return WM_OK;
    seq_scan_args a{};
    a.dtype = dtype; a.T = T; a.N = N; a.H = H;
    if (any) {
        a.gate = *gate; a.x = *x; a.h = *h_seq; a.dh = *dh; a.dgate = *dgate; a.dx = *dx;
    }
    a.h0 = h0; a.reset = reset; a.lengths = lengths; a.dh_last = dh_last; a.dh0 = dh0;
    const wm_status st = reserve(h, wm_seq_scan_ws(h, a, true), s, kWhat);
    if (st != WM_OK) return st;
    return launched(h, wm_seq_scan_launch(h, a, true, s), kWhat);
}

extern "C" wm_status wm_seq_clip(wm_seq *h, int count, const wm_seq_grad *grads, float max_norm, float *norm,
                                 void *cuda_stream) {
    SEQ_BEGIN("wm_seq_clip");
    c.that(count >= 0 && count <= 65536, "0 <= count <= 65536 is needed");
    c.that(count == 0 || grads, "grads is NULL");
    c.that(max_norm >= 0.f, "max_norm must be >= 0");
    c.array(norm, 4, true, "norm is NULL");
    SEQ_CHECKED();
    for (int i = 0; i < count && !c.why; ++i) {
        const wm_seq_grad &g = grads[i];
        c.that(g.n >= 0 && g.n < (1ll << 40), "a gradient's size must be in [0, 2^40)");
        c.that(g.dtype == WM_FP32 || g.dtype == WM_BF16, "dtype must be WM_FP32 or WM_BF16");
        if (c.why) break;
        c.array(g.src, esize(g.dtype), g.n > 0, "a gradient is NULL");
        if (g.dst != g.src) c.array(g.dst, esize(g.dtype), g.n > 0, "a gradient's dst is NULL");
    }
    SEQ_CHECKED();
    const wm_status st = reserve(h, wm_seq_clip_ws(h), s, kWhat);
    if (st != WM_OK) return st;
    return launched(h, wm_seq_clip_launch(h, count, grads, max_norm, norm, s), kWhat);
}
