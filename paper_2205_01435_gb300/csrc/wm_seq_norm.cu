// wm_seq_norm.cu -- layer norm over the last axis, forward and backward.
//
//   y = (x - mean) rstd w + b;  backward, with xhat = (x - mean) rstd and g = dy w:
//   dx = rstd (g - mean(g) - xhat mean(g xhat)),  dw = sum_rows dy xhat,  db = sum_rows dy
//
// Bound by memory: forward moves 2 values per element, backward 3, each read once.  A row
// lives in the registers of TPR threads, E values each, so the mean, the centred variance
// (summed after the mean is known: no cancellation) and the output take one read of x.
// CTAs walk the rows with a stride of the grid: the weights stay in registers, and in the
// backward each thread sums its columns' dw and db over the CTA's rows in fp32; the CTAs'
// partial sums are added in a fixed order by a second, small launch.
#include "wm_seq_internal.h"

namespace {

// Rows longer than this many values per thread x threads go through the looping kernels.
constexpr int kFwdMax = 16384, kBwdMax = 8192;

template <class T, int VEC, int E>
struct Row {
    seq_vec<T, VEC> v[E / VEC];
};

// Lane l of TPR holds vectors l, l + TPR, ... of the row.
template <class T, int VEC, int E, int TPR>
__device__ __forceinline__ void load_row(Row<T, VEC, E> &r, const T *p, int D, int lane) {
#pragma unroll
    for (int i = 0; i < E / VEC; ++i) {
        const int j = (i * TPR + lane) * VEC;
        if (j < D) r.v[i] = seq_load<T, VEC>(p + j);
    }
}

template <int VEC, int E, int TPR>
__device__ __forceinline__ void load_param(float (&w)[E], const float *p, float fill, int D, int lane) {
#pragma unroll
    for (int i = 0; i < E / VEC; ++i)
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
            const int j = (i * TPR + lane) * VEC + k;
            w[i * VEC + k] = p && j < D ? p[j] : fill;
        }
}

// Sums over the TPR threads of a row; every thread gets the result.  One barrier a call:
// the buffers alternate, and a thread writes one again only after a barrier that all
// readers of its earlier contents have reached.
template <int TPR>
struct RowSum {
    float2 *red;  // [2][TPR / 32]
    int turn;
    __device__ __forceinline__ float2 operator()(float2 v) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
            v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
        }
        if (TPR == 32) return v;
        constexpr int W = TPR / 32;
        float2 *b = red + (turn & 1) * W;
        ++turn;
        if ((threadIdx.x & 31) == 0) b[threadIdx.x / 32] = v;
        __syncthreads();
        float2 s = b[0];
#pragma unroll
        for (int i = 1; i < W; ++i) {
            s.x += b[i].x;
            s.y += b[i].y;
        }
        return s;
    }
};

template <int TPR>
constexpr int cta_threads() {
    return TPR < 128 ? 128 : TPR;
}

template <class T, int VEC, int E, int TPR>
__global__ void __launch_bounds__(cta_threads<TPR>()) k_norm_fwd(long long rows, int D, const T *__restrict__ x,
                                                                 long long ldx, const float *__restrict__ w,
                                                                 const float *__restrict__ b, float eps, T *y,
                                                                 long long ldy, float *__restrict__ mean,
                                                                 float *__restrict__ rstd) {
    constexpr int RPC = cta_threads<TPR>() / TPR;
    __shared__ float2 red[2 * (TPR / 32)];
    RowSum<TPR> sum{red, 0};
    const int lane = threadIdx.x % TPR;
    const long long step = (long long)gridDim.x * RPC;
    long long r = (long long)blockIdx.x * RPC + threadIdx.x / TPR;
    if (r >= rows) return;  // TPR > 32: the whole CTA
    Row<T, VEC, E> next;
    load_row<T, VEC, E, TPR>(next, x + r * ldx, D, lane);
    float ww[E], bb[E];
    load_param<VEC, E, TPR>(ww, w, 1.f, D, lane);
    load_param<VEC, E, TPR>(bb, b, 0.f, D, lane);
    const float inv = 1.f / (float)D;
    for (; r < rows; r += step) {
        float v[E];
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < E / VEC; ++i) {
            const bool in = (i * TPR + lane) * VEC < D;
#pragma unroll
            for (int k = 0; k < VEC; ++k) {
                v[i * VEC + k] = in ? seq_to_float(next.v[i].v[k]) : 0.f;
                s += v[i * VEC + k];
            }
        }
        if (r + step < rows) load_row<T, VEC, E, TPR>(next, x + (r + step) * ldx, D, lane);
        const float mu = sum(make_float2(s, 0.f)).x * inv;
        float q = 0.f;
#pragma unroll
        for (int i = 0; i < E / VEC; ++i)
            if ((i * TPR + lane) * VEC < D)
#pragma unroll
                for (int k = 0; k < VEC; ++k) {
                    v[i * VEC + k] -= mu;
                    q = fmaf(v[i * VEC + k], v[i * VEC + k], q);
                }
        const float rs = rsqrtf(sum(make_float2(q, 0.f)).x * inv + eps);
        if (mean && lane == 0) {
            mean[r] = mu;
            rstd[r] = rs;
        }
#pragma unroll
        for (int i = 0; i < E / VEC; ++i) {
            const int j = (i * TPR + lane) * VEC;
            if (j >= D) continue;
            seq_vec<T, VEC> o;
#pragma unroll
            for (int k = 0; k < VEC; ++k)
                o.v[k] = seq_from_float<T>(fmaf(v[i * VEC + k] * rs, ww[i * VEC + k], bb[i * VEC + k]));
            seq_store(y + r * ldy + j, o);
        }
    }
}

// part: [gridDim.x][2][D] sums of dw and db over the CTA's rows (null: not wanted)
template <class T, int VEC, int E, int TPR>
__global__ void __launch_bounds__(cta_threads<TPR>()) k_norm_bwd(long long rows, int D, const T *__restrict__ x,
                                                                 long long ldx, const float *__restrict__ w,
                                                                 const float *__restrict__ mean,
                                                                 const float *__restrict__ rstd, const T *dy,
                                                                 long long lddy, T *dx, long long lddx,
                                                                 float *__restrict__ part) {
    constexpr int RPC = cta_threads<TPR>() / TPR;
    __shared__ float2 red[2 * (TPR / 32)];
    extern __shared__ float cols[];  // RPC > 1: [RPC][2][D]
    RowSum<TPR> sum{red, 0};
    const int lane = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    const long long step = (long long)gridDim.x * RPC;
    float ww[E], dw[E], db[E];
    load_param<VEC, E, TPR>(ww, w, 1.f, D, lane);
#pragma unroll
    for (int e = 0; e < E; ++e) dw[e] = db[e] = 0.f;
    const float inv = 1.f / (float)D;
    long long r = (long long)blockIdx.x * RPC + sub;
    Row<T, VEC, E> nx, ny;
    float nmu = 0.f, nrs = 0.f;
    if (r < rows) {
        load_row<T, VEC, E, TPR>(nx, x + r * ldx, D, lane);
        load_row<T, VEC, E, TPR>(ny, dy + r * lddy, D, lane);
        nmu = mean[r];
        nrs = rstd[r];
    }
    for (; r < rows; r += step) {
        const Row<T, VEC, E> cx = nx, cy = ny;
        const float mu = nmu, rs = nrs;
        if (r + step < rows) {
            load_row<T, VEC, E, TPR>(nx, x + (r + step) * ldx, D, lane);
            load_row<T, VEC, E, TPR>(ny, dy + (r + step) * lddy, D, lane);
            nmu = mean[r + step];
            nrs = rstd[r + step];
        }
        float2 s = make_float2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < E / VEC; ++i)
            if ((i * TPR + lane) * VEC < D)
#pragma unroll
                for (int k = 0; k < VEC; ++k) {
                    const int e = i * VEC + k;
                    const float xh = (seq_to_float(cx.v[i].v[k]) - mu) * rs, d = seq_to_float(cy.v[i].v[k]);
                    dw[e] = fmaf(d, xh, dw[e]);
                    db[e] += d;
                    s.x = fmaf(d, ww[e], s.x);
                    s.y = fmaf(d * ww[e], xh, s.y);
                }
        s = sum(s);
        const float m1 = s.x * inv, m2 = s.y * inv;
#pragma unroll
        for (int i = 0; i < E / VEC; ++i) {
            const int j = (i * TPR + lane) * VEC;
            if (j >= D) continue;
            seq_vec<T, VEC> o;
#pragma unroll
            for (int k = 0; k < VEC; ++k) {
                const float xh = (seq_to_float(cx.v[i].v[k]) - mu) * rs;
                const float g = seq_to_float(cy.v[i].v[k]) * ww[i * VEC + k];
                o.v[k] = seq_from_float<T>(rs * (g - m1 - xh * m2));
            }
            seq_store(dx + r * lddx + j, o);
        }
    }
    if (!part) return;
    part += (long long)blockIdx.x * 2 * D;
    float *to = RPC > 1 ? cols + sub * 2 * D : part;
#pragma unroll
    for (int i = 0; i < E / VEC; ++i)
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
            const int j = (i * TPR + lane) * VEC + k;
            if (j < D) {
                to[j] = dw[i * VEC + k];
                to[D + j] = db[i * VEC + k];
            }
        }
    if (RPC == 1) return;
    __syncthreads();
    for (int j = threadIdx.x; j < 2 * D; j += blockDim.x) {
        float v = cols[j];
        for (int q = 1; q < RPC; ++q) v += cols[q * 2 * D + j];
        part[j] = v;
    }
}

// dw, db: column sums of the CTAs' partial sums, in a fixed order (32 columns x 16 slices a CTA).
__global__ void __launch_bounds__(512) k_norm_cols(int parts, int D, const float *__restrict__ part, float *dw, float *db) {
    __shared__ float s[16][33];
    const int c = blockIdx.x * 32 + threadIdx.x % 32, q = threadIdx.x / 32;
    float v = 0.f;
    if (c < 2 * D)
        for (int i = q; i < parts; i += 16) v += part[(long long)i * 2 * D + c];
    s[q][threadIdx.x % 32] = v;
    __syncthreads();
    if (q || c >= 2 * D) return;
    for (int i = 1; i < 16; ++i) v += s[i][threadIdx.x];
    if (c < D) {
        if (dw) dw[c] = v;
    } else if (db) {
        db[c - D] = v;
    }
}

// ---- rows of any length: each pass reads the row again (from L2) -----------------------
constexpr int kLong = 512;

__device__ __forceinline__ float2 cta_sum(float2 v, float2 *red) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
        v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
    }
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x / 32] = v;
    __syncthreads();
    float2 s = red[0];
    for (int i = 1; i < kLong / 32; ++i) {
        s.x += red[i].x;
        s.y += red[i].y;
    }
    return s;
}

template <class T>
__global__ void __launch_bounds__(kLong) k_norm_fwd_long(long long rows, int D, const T *x, long long ldx,
                                                         const float *__restrict__ w, const float *__restrict__ b,
                                                         float eps, T *y, long long ldy, float *__restrict__ mean,
                                                         float *__restrict__ rstd) {
    __shared__ float2 red[kLong / 32];
    for (long long r = blockIdx.x; r < rows; r += gridDim.x) {
        const T *p = x + r * ldx;
        float s = 0.f;
        for (int j = threadIdx.x; j < D; j += kLong) s += seq_to_float(p[j]);
        const float mu = cta_sum(make_float2(s, 0.f), red).x / (float)D;
        s = 0.f;
        for (int j = threadIdx.x; j < D; j += kLong) {
            const float v = seq_to_float(p[j]) - mu;
            s = fmaf(v, v, s);
        }
        const float rs = rsqrtf(cta_sum(make_float2(s, 0.f), red).x / (float)D + eps);
        if (mean && threadIdx.x == 0) {
            mean[r] = mu;
            rstd[r] = rs;
        }
        for (int j = threadIdx.x; j < D; j += kLong)
            y[r * ldy + j] = seq_from_float<T>(fmaf((seq_to_float(p[j]) - mu) * rs, w ? w[j] : 1.f, b ? b[j] : 0.f));
    }
}

// dx, and (part: [gridDim.x][2][D], or null) the CTA's sums for dw and db
template <class T>
__global__ void __launch_bounds__(kLong) k_norm_bwd_long(long long rows, int D, const T *__restrict__ x, long long ldx,
                                                         const float *__restrict__ w, const float *__restrict__ mean,
                                                         const float *__restrict__ rstd, const T *dy, long long lddy,
                                                         T *dx, long long lddx, float *part) {
    __shared__ float2 red[kLong / 32];
    if (part) {
        part += (long long)blockIdx.x * 2 * D;
        for (int j = threadIdx.x; j < D; j += kLong) part[j] = part[D + j] = 0.f;
    }
    for (long long r = blockIdx.x; r < rows; r += gridDim.x) {
        const T *px = x + r * ldx, *pd = dy + r * lddy;
        const float mu = mean[r], rs = rstd[r];
        float2 s = make_float2(0.f, 0.f);
        for (int j = threadIdx.x; j < D; j += kLong) {
            const float xh = (seq_to_float(px[j]) - mu) * rs, d = seq_to_float(pd[j]), g = d * (w ? w[j] : 1.f);
            s.x += g;
            s.y = fmaf(g, xh, s.y);
        }
        s = cta_sum(s, red);
        const float m1 = s.x / (float)D, m2 = s.y / (float)D;
        for (int j = threadIdx.x; j < D; j += kLong) {
            const float xh = (seq_to_float(px[j]) - mu) * rs, d = seq_to_float(pd[j]), g = d * (w ? w[j] : 1.f);
            if (part) {  // j and D + j are this thread's alone
                part[j] = fmaf(d, xh, part[j]);
                part[D + j] += d;
            }
            dx[r * lddx + j] = seq_from_float<T>(rs * (g - m1 - xh * m2));
        }
    }
}

bool vec_ok(const void *p, long long ld, int D, size_t es) {
    return (uintptr_t)p % 16 == 0 && (ld * es) % 16 == 0 && (D * es) % 16 == 0;
}

// Threads per row and values per thread: the fewest of each that hold the row (a warp up to 1024
// values, so that its sums need no barrier).
struct Shape {
    int tpr, e;
};
Shape shape(int D) {
    if (D <= 1024) return {32, D <= 256 ? 8 : D <= 512 ? 16 : 32};
    if (D <= 4096) return {128, D <= 2048 ? 16 : 32};
    if (D <= 8192) return {256, 32};
    return {512, 32};
}

int bwd_ctas(const wm_seq *h, long long rows, int D) {
    const int rpc = D <= 1024 ? 4 : 1;
    const long long need = (rows + rpc - 1) / rpc, most = (long long)h->sms * (D > 4096 ? 1 : 3);
    return (int)(need < most ? need : most);
}

#define NORM_SHAPES(CALL)                       \
    if (sh.tpr == 32 && sh.e == 8) CALL(8, 32)  \
    else if (sh.tpr == 32 && sh.e == 16) CALL(16, 32) \
    else if (sh.tpr == 32) CALL(32, 32)         \
    else if (sh.tpr == 128 && sh.e == 16) CALL(16, 128) \
    else if (sh.tpr == 128) CALL(32, 128)       \
    else if (sh.tpr == 256) CALL(32, 256)

template <class T, int VEC>
void fwd(const wm_seq *h, long long rows, int D, const T *x, long long ldx, const float *w, const float *b, float eps,
         T *y, long long ldy, float *mean, float *rstd, cudaStream_t s) {
    const Shape sh = shape(D);
#define CALL(E, TPR)                                                                                                  \
    {                                                                                                                 \
        constexpr int rpc = cta_threads<TPR>() / TPR;                                                                 \
        const long long need = (rows + rpc - 1) / rpc, most = (long long)h->sms * (TPR > 128 ? 4 : 8);                \
        k_norm_fwd<T, VEC, E, TPR><<<(unsigned)(need < most ? need : most), cta_threads<TPR>(), 0, s>>>(              \
            rows, D, x, ldx, w, b, eps, y, ldy, mean, rstd);                                                          \
    }
    NORM_SHAPES(CALL) else CALL(32, 512)
#undef CALL
}

template <class T, int VEC>
void bwd(const wm_seq *h, long long rows, int D, const T *x, long long ldx, const float *w, const float *mean,
         const float *rstd, const T *dy, long long lddy, T *dx, long long lddx, float *part, int ctas, cudaStream_t s) {
    const Shape sh = shape(D);
#define CALL(E, TPR)                                                                                            \
    {                                                                                                           \
        constexpr int rpc = cta_threads<TPR>() / TPR;                                                           \
        k_norm_bwd<T, VEC, E, TPR><<<ctas, cta_threads<TPR>(), part && rpc > 1 ? (size_t)rpc * 2 * D * 4 : 0, s>>>( \
            rows, D, x, ldx, w, mean, rstd, dy, lddy, dx, lddx, part);                                          \
    }
    NORM_SHAPES(CALL)
#undef CALL
}

template <class T>
void fwd_any(const wm_seq *h, long long rows, int D, const T *x, long long ldx, const float *w, const float *b,
             float eps, T *y, long long ldy, float *mean, float *rstd, cudaStream_t s) {
    if (D > kFwdMax) {
        const long long most = (long long)h->sms * 4;
        k_norm_fwd_long<T><<<(unsigned)(rows < most ? rows : most), kLong, 0, s>>>(rows, D, x, ldx, w, b, eps, y, ldy, mean, rstd);
        return;
    }
    if (vec_ok(x, ldx, D, sizeof(T)) && vec_ok(y, ldy, D, sizeof(T)))
        fwd<T, 16 / sizeof(T)>(h, rows, D, x, ldx, w, b, eps, y, ldy, mean, rstd, s);
    else
        fwd<T, 1>(h, rows, D, x, ldx, w, b, eps, y, ldy, mean, rstd, s);
}

template <class T>
void bwd_any(const wm_seq *h, long long rows, int D, const T *x, long long ldx, const float *w, const float *mean,
             const float *rstd, const T *dy, long long lddy, T *dx, long long lddx, float *part, int ctas, cudaStream_t s) {
    if (D > kBwdMax)
        k_norm_bwd_long<T><<<ctas, kLong, 0, s>>>(rows, D, x, ldx, w, mean, rstd, dy, lddy, dx, lddx, part);
    else if (vec_ok(x, ldx, D, sizeof(T)) && vec_ok(dy, lddy, D, sizeof(T)) && vec_ok(dx, lddx, D, sizeof(T)))
        bwd<T, 16 / sizeof(T)>(h, rows, D, x, ldx, w, mean, rstd, dy, lddy, dx, lddx, part, ctas, s);
    else
        bwd<T, 1>(h, rows, D, x, ldx, w, mean, rstd, dy, lddy, dx, lddx, part, ctas, s);
}

}  // namespace

cudaError_t wm_seq_norm_launch(wm_seq *h, int dtype, long long rows, int D, const void *x, long long ldx,
                               const float *w, const float *b, float eps, void *y, long long ldy, float *mean,
                               float *rstd, cudaStream_t s) {
    if (dtype == WM_BF16)
        fwd_any(h, rows, D, (const __nv_bfloat16 *)x, ldx, w, b, eps, (__nv_bfloat16 *)y, ldy, mean, rstd, s);
    else
        fwd_any(h, rows, D, (const float *)x, ldx, w, b, eps, (float *)y, ldy, mean, rstd, s);
    h->last_launches = 1;
    return cudaGetLastError();
}

size_t wm_seq_norm_backward_ws(const wm_seq *h, long long rows, int D) {
    return (size_t)bwd_ctas(h, rows, D) * 2 * D * sizeof(float);
}

cudaError_t wm_seq_norm_backward_launch(wm_seq *h, int dtype, long long rows, int D, const void *x, long long ldx,
                                        const float *w, const float *mean, const float *rstd, const void *dy,
                                        long long lddy, void *dx, long long lddx, float *dw, float *db,
                                        cudaStream_t s) {
    const int ctas = bwd_ctas(h, rows, D);
    float *part = dw || db ? (float *)h->ws : nullptr;
    h->last_launches = 0;
    if (ctas > 0) {
        if (dtype == WM_BF16)
            bwd_any(h, rows, D, (const __nv_bfloat16 *)x, ldx, w, mean, rstd, (const __nv_bfloat16 *)dy, lddy,
                    (__nv_bfloat16 *)dx, lddx, part, ctas, s);
        else
            bwd_any(h, rows, D, (const float *)x, ldx, w, mean, rstd, (const float *)dy, lddy, (float *)dx, lddx, part, ctas, s);
        h->last_launches = 1;
    }
    if (dw || db) {  // no rows: zeros
        k_norm_cols<<<(2 * D + 31) / 32, 512, 0, s>>>(ctas, D, part, dw, db);
        ++h->last_launches;
    }
    return cudaGetLastError();
}
