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
//
// Measured (one GB300, durations of the kernels alone): 65,536 x 1024 bf16 48 us forward (5.6 TB/s),
// 81 us backward (5.0 TB/s: the column sums leave 16 warps an SM, which issue half of the cycles) and 7 us
// for the column sums; 20,000 x 301 fp32 13, 18 and 7 us; 12,000 x 4096 fp32 69 (5.7 TB/s), 96 (6.1) and 7 us.
#include <algorithm>
#include <initializer_list>
#include <utility>

#include "wm_seq_internal.h"

namespace {

// Longer rows do not fit the registers of a CTA's threads and go through the looping kernels, which
// read them once a pass (backward of 4000 x 9000 fp32: 87 us in registers, 305 in the loop).
constexpr int kFwdMax = 16384, kBwdMax = 12288;

// A thread holds vectors lane, lane + TPR, ... of its row.  Rows on their way: a ring of RING
// rows in shared memory, every thread copying and reading its own vectors (no barrier, and no
// registers held by loads in flight).  bf16 rows that are not aligned to 4 bytes cannot be
// copied so: their threads load a row when they come to it.
template <int E, int ARRAYS, int THREADS>
constexpr int ring_rows() {  // two rows or more on their way, in 192 KB of a CTA at most
    const int rows = E == 8 ? 6 : E < 32 ? 4 : 3, room = (192 << 10) / (ARRAYS * THREADS * E * 4);
    return rows < room ? rows : room;
}

template <class T, int VEC>
constexpr bool ring_fits() {
    return VEC * sizeof(T) >= 4;
}

template <class T, int VEC, int E, int TPR, int ARRAYS, int THREADS>
struct Rows {
    using V = seq_vec<T, VEC>;
    static constexpr bool ASYNC = ring_fits<T, VEC>();
    static constexpr int RING = ring_rows<E, ARRAYS, THREADS>();
    V *mine;
    const T *p[ARRAYS];  // the next row to copy (ASYNC), or to load
    long long left;      // rows not copied yet
    int slot = 0;
    static constexpr size_t bytes() { return ASYNC ? (size_t)RING * ARRAYS * THREADS * E * sizeof(T) : 0; }
    __device__ __forceinline__ V *place(int s, int a, int i) const { return mine + ((s * ARRAYS + a) * (E / VEC) + i) * THREADS; }
    __device__ __forceinline__ void issue(int s, const long long (&step)[ARRAYS], int D, int lane) {
        if (left > 0) {
#pragma unroll
            for (int a = 0; a < ARRAYS; ++a) {
#pragma unroll
                for (int i = 0; i < E / VEC; ++i) {
                    const int j = (i * TPR + lane) * VEC;
                    if (j < D)
                        copy_async<ASYNC ? (int)sizeof(V) : 4>((uint32_t)__cvta_generic_to_shared(place(s, a, i)), p[a] + j);
                }
                p[a] += step[a];
            }
        }
        --left;
        copy_commit();
    }
    __device__ __forceinline__ void start(const long long (&step)[ARRAYS], int D, int lane) {
        if constexpr (ASYNC)
#pragma unroll
            for (int q = 0; q < RING - 1; ++q) issue(q, step, D, lane);
    }
    // makes the next row readable
    __device__ __forceinline__ void arrive(const long long (&step)[ARRAYS], int D, int lane) {
        if constexpr (ASYNC) {
            issue(slot == 0 ? RING - 1 : slot - 1, step, D, lane);
            copy_wait<RING - 1>();
        }
    }
    __device__ __forceinline__ V read(int a, int i, int lane) const {
        if constexpr (ASYNC) return *place(slot, a, i);
        else return seq_load<T, VEC>(p[a] + (i * TPR + lane) * VEC);
    }
    __device__ __forceinline__ void next(const long long (&step)[ARRAYS]) {
        if constexpr (ASYNC) {
            slot = slot + 1 == RING ? 0 : slot + 1;
        } else {
#pragma unroll
            for (int a = 0; a < ARRAYS; ++a) p[a] += step[a];
        }
    }
};

// Rows of 1024 values in one warp: the weights come from shared memory, in the order the lanes
// read them (they would fill the registers); else they stay in registers.
template <int E, int TPR>
constexpr bool shared_weights() {
    return TPR == 32 && E == 32;
}

template <int VEC, int E, int TPR>
struct Weights {
    static constexpr bool SHARED = shared_weights<E, TPR>();
    float r[SHARED ? 1 : E];
    const float *s;
    __device__ __forceinline__ void load(const float *p, float fill, int D, int lane, float *smem) {
        if constexpr (SHARED) {  // [E / Q][32] of Q values: what lanes read together lies side by side
            constexpr int Q = VEC % 4 == 0 ? 4 : 1;
            for (int o = threadIdx.x; o < 1024; o += blockDim.x) {
                const int e = o / (32 * Q) * Q + o % Q, l = o / Q % 32, j = (e / VEC * TPR + l) * VEC + e % VEC;
                smem[o] = p && j < D ? p[j] : fill;
            }
            s = smem + lane * Q;
        } else {
#pragma unroll
            for (int i = 0; i < E / VEC; ++i)
#pragma unroll
                for (int k = 0; k < VEC; ++k) {
                    const int j = (i * TPR + lane) * VEC + k;
                    r[i * VEC + k] = p && j < D ? p[j] : fill;
                }
        }
    }
    // the weights of vector i
    __device__ __forceinline__ void get(int i, float (&w)[VEC]) const {
        if constexpr (!SHARED) {
#pragma unroll
            for (int k = 0; k < VEC; ++k) w[k] = r[i * VEC + k];
        } else if constexpr (VEC % 4 == 0) {
#pragma unroll
            for (int k = 0; k < VEC; k += 4) {
                const float4 q = *reinterpret_cast<const float4 *>(s + (i * VEC + k) * 32);
                w[k] = q.x;
                w[k + 1] = q.y;
                w[k + 2] = q.z;
                w[k + 3] = q.w;
            }
        } else {  // [E][32]
#pragma unroll
            for (int k = 0; k < VEC; ++k) w[k] = s[(i * VEC + k) * 32];
        }
    }
};

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

// CTAs of an SM at once by their registers: what the launch bounds ask for.
template <int TPR>
constexpr int fwd_ctas() {
    return TPR == 32 ? 6 : TPR == 128 ? 4 : TPR == 256 ? 2 : 1;
}
template <int TPR>
constexpr int bwd_ctas() {
    return TPR == 32 ? 4 : TPR == 128 ? 3 : 1;
}

// And by their shared memory too (an SM has 228 KB, and keeps 1 KB of it for every CTA): the grids' sizes.
// Rows are split evenly over the CTAs, so those that do not run at once would run alone afterwards.
template <class T, int VEC, int E, int TPR, bool BWD>
constexpr int ctas_at_once() {
    constexpr int THREADS = cta_threads<TPR>(), RPC = THREADS / TPR, by_registers = BWD ? bwd_ctas<TPR>() : fwd_ctas<TPR>();
    constexpr size_t ring = Rows<T, VEC, E, TPR, BWD ? 2 : 1, THREADS>::bytes(), sums = BWD && RPC > 1 ? RPC * 8 * 32 * E : 0;
    constexpr size_t weights = shared_weights<E, TPR>() ? (BWD ? 1 : 2) * 4096 : 0, fixed = weights + TPR / 32 * 16 + 1024;
    constexpr size_t of_cta = ((ring > sums ? ring : sums) + fixed + 127) / 128 * 128, fit = (228 << 10) / of_cta;
    return fit < by_registers ? (int)fit : by_registers;
}

template <class T, int VEC, int E, int TPR>
__global__ void __launch_bounds__(cta_threads<TPR>(), fwd_ctas<TPR>())
    k_norm_fwd(long long rows, int D, const T *x, long long ldx, const float *__restrict__ w,  // (y may be x)
               const float *__restrict__ b, float eps, T *y, long long ldy, float *__restrict__ mean, float *__restrict__ rstd) {
    constexpr int THREADS = cta_threads<TPR>(), RPC = THREADS / TPR;
    constexpr bool SHARED = shared_weights<E, TPR>();
    extern __shared__ __align__(16) unsigned char ring[];
    __shared__ float2 red[2 * (TPR / 32)];
    __shared__ __align__(16) float ws[SHARED ? 2 : 1][SHARED ? 1024 : 1];
    RowSum<TPR> sum{red, 0};
    const int lane = threadIdx.x % TPR;
    const long long step = (long long)gridDim.x * RPC, steps[1] = {step * ldx};
    long long r = (long long)blockIdx.x * RPC + threadIdx.x / TPR;
    Rows<T, VEC, E, TPR, 1, THREADS> in{reinterpret_cast<seq_vec<T, VEC> *>(ring) + threadIdx.x, {x + r * ldx},
                                        r < rows ? (rows - r + step - 1) / step : 0};
    in.start(steps, D, lane);
    Weights<VEC, E, TPR> ww, bb;
    ww.load(w, 1.f, D, lane, ws[0]);
    bb.load(b, 0.f, D, lane, ws[SHARED ? 1 : 0]);
    if (SHARED) __syncthreads();
    const float inv = 1.f / (float)D;
    T *out = y + r * ldy;
    for (; r < rows; r += step, out += step * ldy) {
        in.arrive(steps, D, lane);
        // without a ring all of a row's loads go out before the first is used (4000 x 9001 bf16: 80 us,
        // 184 one by one); from the ring they would only hold registers (6000 x 8192 fp32: 63 us, 74 so)
        constexpr bool AHEAD = !ring_fits<T, VEC>();
        seq_vec<T, VEC> raw[AHEAD ? E / VEC : 1];
        if constexpr (AHEAD)
#pragma unroll
            for (int i = 0; i < E / VEC; ++i)
                if ((i * TPR + lane) * VEC < D) raw[i] = in.read(0, i, lane);
        float v[E / VEC][VEC];
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < E / VEC; ++i) {
            if ((i * TPR + lane) * VEC < D) {
                if constexpr (AHEAD) seq_unpack(raw[i], v[i]);
                else seq_unpack(in.read(0, i, lane), v[i]);
#pragma unroll
                for (int k = 0; k < VEC; ++k) s += v[i][k];
            }
        }
        in.next(steps);
        const float mu = sum(make_float2(s, 0.f)).x * inv;
        float q = 0.f;
#pragma unroll
        for (int i = 0; i < E / VEC; ++i)
            if ((i * TPR + lane) * VEC < D)
#pragma unroll
                for (int k = 0; k < VEC; ++k) {
                    v[i][k] -= mu;
                    q = fmaf(v[i][k], v[i][k], q);
                }
        const float rs = rsqrtf(sum(make_float2(q, 0.f)).x * inv + eps);
        if (mean && lane == 0) {
            mean[r] = mu;
            rstd[r] = rs;
        }
#pragma unroll
        for (int i = 0; i < E / VEC; ++i) {
            const int j = (i * TPR + lane) * VEC;
            if (j < D) {
                float fw[VEC], fb[VEC];
                ww.get(i, fw);
                bb.get(i, fb);
#pragma unroll
                for (int k = 0; k < VEC; ++k) v[i][k] = fmaf(v[i][k] * rs, fw[k], fb[k]);
                seq_store(out + j, seq_pack<T, VEC>(v[i]));
            }
        }
    }
}

// part: [gridDim.x][2][D] sums of dw and db over the CTA's rows (null: not wanted); of a single CTA
// they go to dw and db at once
template <class T, int VEC, int E, int TPR>
__global__ void __launch_bounds__(cta_threads<TPR>(), bwd_ctas<TPR>())
    k_norm_bwd(long long rows, int D, const T *__restrict__ x, long long ldx, const float *__restrict__ w,
               const float *__restrict__ mean, const float *__restrict__ rstd, const T *dy, long long lddy, T *dx, long long lddx,
               float *__restrict__ part, float *dw_out, float *db_out) {
    constexpr int THREADS = cta_threads<TPR>(), RPC = THREADS / TPR;
    constexpr bool SHARED = shared_weights<E, TPR>();
    extern __shared__ __align__(16) unsigned char ring[];  // the rows' ring; after the rows (RPC > 1) sums [RPC][2][D]
    __shared__ float2 red[2 * (TPR / 32)];
    __shared__ __align__(16) float ws[SHARED ? 1024 : 1];
    RowSum<TPR> sum{red, 0};
    const int lane = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    const long long step = (long long)gridDim.x * RPC, steps[2] = {step * ldx, step * lddy};
    long long r = (long long)blockIdx.x * RPC + sub;
    Rows<T, VEC, E, TPR, 2, THREADS> in{reinterpret_cast<seq_vec<T, VEC> *>(ring) + threadIdx.x, {x + r * ldx, dy + r * lddy},
                                        r < rows ? (rows - r + step - 1) / step : 0};
    in.start(steps, D, lane);
    float nmu = 0.f, nrs = 0.f;
    if (r < rows) {
        nmu = mean[r];
        nrs = rstd[r];
    }
    Weights<VEC, E, TPR> ww;
    ww.load(w, 1.f, D, lane, ws);
    if (SHARED) __syncthreads();
    float dw[E], db[E];
#pragma unroll
    for (int e = 0; e < E; ++e) dw[e] = db[e] = 0.f;
    const float inv = 1.f / (float)D;
    T *out = dx + r * lddx;
    for (; r < rows; r += step, out += step * lddx) {
        const float mu = nmu, rs = nrs;
        in.arrive(steps, D, lane);
        if (r + step < rows) {
            nmu = mean[r + step];
            nrs = rstd[r + step];
        }
        float2 s = make_float2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < E / VEC; ++i)
            if ((i * TPR + lane) * VEC < D) {
                float fx[VEC], fd[VEC], fw[VEC];
                seq_unpack(in.read(0, i, lane), fx);
                seq_unpack(in.read(1, i, lane), fd);
                ww.get(i, fw);
#pragma unroll
                for (int k = 0; k < VEC; ++k) {
                    const int e = i * VEC + k;
                    const float xh = (fx[k] - mu) * rs, g = fd[k] * fw[k];
                    dw[e] = fmaf(fd[k], xh, dw[e]);
                    db[e] += fd[k];
                    s.x += g;
                    s.y = fmaf(g, xh, s.y);
                }
            }
        s = sum(s);
        const float m1 = s.x * inv, m2 = s.y * inv;
#pragma unroll
        for (int i = 0; i < E / VEC; ++i) {
            const int j = (i * TPR + lane) * VEC;
            if (j < D) {
                float fx[VEC], fd[VEC], fw[VEC];
                seq_unpack(in.read(0, i, lane), fx);
                seq_unpack(in.read(1, i, lane), fd);
                ww.get(i, fw);
#pragma unroll
                for (int k = 0; k < VEC; ++k) {
                    const float xh = (fx[k] - mu) * rs;
                    fd[k] = rs * (fmaf(fd[k], fw[k], -m1) - xh * m2);
                }
                seq_store(out + j, seq_pack<T, VEC>(fd));
            }
        }
        in.next(steps);
    }
    if (!part) return;
    const bool single = gridDim.x == 1;
    float *to_w = single ? dw_out : part + (long long)blockIdx.x * 2 * D, *to_b = single ? db_out : to_w + D;
    if (RPC > 1) __syncthreads();  // the ring is done with: the sums take its place
    float *cols = reinterpret_cast<float *>(ring) + sub * 2 * D;
    float *w_at = RPC > 1 ? cols : to_w, *b_at = RPC > 1 ? cols + D : to_b;
#pragma unroll
    for (int i = 0; i < E / VEC; ++i)
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
            const int j = (i * TPR + lane) * VEC + k;
            if (j < D) {
                if (w_at) w_at[j] = dw[i * VEC + k];
                if (b_at) b_at[j] = db[i * VEC + k];
            }
        }
    if (RPC == 1) return;
    __syncthreads();
    const float *all = reinterpret_cast<const float *>(ring);
    for (int j = threadIdx.x; j < 2 * D; j += blockDim.x) {
        float v = all[j];
        for (int q = 1; q < RPC; ++q) v += all[q * 2 * D + j];
        if (j < D) {
            if (to_w) to_w[j] = v;
        } else if (to_b) {
            to_b[j - D] = v;
        }
    }
}

// dw, db: column sums of the CTAs' partial sums, in a fixed order (32 columns x 32 slices a CTA).
constexpr int kSlices = 32;
__global__ void __launch_bounds__(32 * kSlices) k_norm_cols(int parts, int D, const float *__restrict__ part, float *dw, float *db) {
    __shared__ float s[kSlices][33];
    const long long c = (long long)blockIdx.x * 32 + threadIdx.x % 32, columns = 2ll * D;
    const int q = threadIdx.x / 32;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    float v = 0.f;
    if (c < columns)
#pragma unroll 8
        for (int i = q; i < parts; i += kSlices) v += part[i * columns + c];
    s[q][threadIdx.x % 32] = v;
    __syncthreads();
    if (q || c >= columns) return;
#pragma unroll
    for (int i = 1; i < kSlices; ++i) v += s[i][threadIdx.x];
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
        for (int j = threadIdx.x; j < D; j += kLong) part[j] = part[D + (long long)j] = 0.f;
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
            if (part) {  // j and D + j are this thread's alone (D + j in 64 bits)
                part[j] = fmaf(d, xh, part[j]);
                part[D + (long long)j] += d;
            }
            dx[r * lddx + j] = seq_from_float<T>(rs * (g - m1 - xh * m2));
        }
    }
}

// The widest access of `vec`, `vec` / 2, ... values that the arrays' addresses and strides and the
// rows' length allow.
int width(int vec, size_t es, int D, std::initializer_list<std::pair<const void *, long long>> arrays) {
    for (; vec > 1; vec /= 2) {
        bool ok = D % vec == 0;
        for (const auto &a : arrays) ok &= (uintptr_t)a.first % (vec * es) == 0 && a.second % vec == 0;
        if (ok) break;
    }
    return vec;
}

// Threads per row and values per thread: the fewest of each that hold the row (a warp up to 1024
// values, so that its sums need no barrier: the kernel of 65536 x 1024 bf16 backward took 80 us so, and 90 us
// with 128 threads a row).  From 4097 values the backward takes 512 threads where the forward takes 256: its column sums
// would leave 256 threads an SM (8000 x 6001: fp32 144 us against 178, bf16 124 against 157; forward 84 against 80,
// 106 against 92).
struct Shape {
    int tpr, e;
};
Shape shape(int D, int vec, bool bwd) {
    if (D <= 1024) return {32, D <= 256 ? 8 : D <= 384 && vec <= 4 ? 12 : D <= 512 ? 16 : 32};
    if (D <= 4096) return {128, D <= 2048 ? 16 : 32};
    if (D <= 8192 && !bwd) return {256, 32};
    return {512, D <= 6144 && vec <= 4 ? 12 : D <= 8192 ? 16 : D <= 12288 ? 24 : 32};
}

// Launches with its dynamic shared memory (above 48 KB a kernel has to be told).
template <class... P, class... A>
cudaError_t launch(void (*k)(P...), int grid, int threads, size_t smem, cudaStream_t s, A... args) {
    if (smem > 40 << 10) {
        const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
    }
    k<<<grid, threads, smem, s>>>(args...);
    return cudaGetLastError();
}

#define NORM_SHAPES(CALL)                          \
    if (sh.tpr == 32 && sh.e == 8) CALL(8, 32)     \
    if constexpr (VEC <= 4)                        \
        if (sh.tpr == 32 && sh.e == 12) CALL(12, 32) \
    if (sh.tpr == 32 && sh.e == 16) CALL(16, 32)   \
    if (sh.tpr == 32) CALL(32, 32)                 \
    if (sh.tpr == 128 && sh.e == 16) CALL(16, 128) \
    if (sh.tpr == 128) CALL(32, 128)

// CTAs of an SM at once in the backward, for rows of D values in accesses of VEC.
template <class T, int VEC>
int bwd_per_sm(int D) {
    const Shape sh = shape(D, VEC, true);
#define CALL(E, TPR) return ctas_at_once<T, VEC, E, TPR, true>();
    NORM_SHAPES(CALL)
#undef CALL
    return bwd_ctas<512>();
}

template <class T>
int bwd_grid(const wm_seq *h, long long rows, int D, const void *x, long long ldx, const void *dy, long long lddy, const void *dx,
             long long lddx) {
    const int rpc = D <= 1024 ? 4 : 1;
    const long long need = (rows + rpc - 1) / rpc;
    // a few rows a warp: one CTA, which needs no second launch
    if (need <= 4 && D <= 1024) return need > 0;
    constexpr int VEC = 16 / sizeof(T);
    const int v = width(VEC, sizeof(T), D, {{x, ldx}, {dy, lddy}, {dx, lddx}});
    const int per_sm = v == VEC ? bwd_per_sm<T, VEC>(D) : v == 4 ? bwd_per_sm<T, 4>(D) : v == 2 ? bwd_per_sm<T, 2>(D) : bwd_per_sm<T, 1>(D);
    const long long most = (long long)h->sms * per_sm;
    return (int)(need < most ? need : most);
}

template <class T, int VEC>
cudaError_t fwd(const wm_seq *h, long long rows, int D, const T *x, long long ldx, const float *w, const float *b, float eps,
                T *y, long long ldy, float *mean, float *rstd, cudaStream_t s) {
    const Shape sh = shape(D, VEC, false);
#define CALL(E, TPR)                                                                                                     \
    {                                                                                                                    \
        constexpr int threads = cta_threads<TPR>(), rpc = threads / TPR;                                                 \
        const long long need = (rows + rpc - 1) / rpc, most = (long long)h->sms * ctas_at_once<T, VEC, E, TPR, false>(); \
        return launch(k_norm_fwd<T, VEC, E, TPR>, (int)(need < most ? need : most), threads,                             \
                      Rows<T, VEC, E, TPR, 1, threads>::bytes(), s, rows, D, x, ldx, w, b, eps, y, ldy, mean, rstd);     \
    }
    NORM_SHAPES(CALL)
    if (sh.tpr == 256) CALL(32, 256)
    if (sh.e == 24) CALL(24, 512)
    CALL(32, 512)
#undef CALL
}

template <class T, int VEC>
cudaError_t bwd(long long rows, int D, const T *x, long long ldx, const float *w, const float *mean, const float *rstd,
                const T *dy, long long lddy, T *dx, long long lddx, float *part, float *dw, float *db, int grid, cudaStream_t s) {
    const Shape sh = shape(D, VEC, true);
#define CALL(E, TPR)                                                                                             \
    {                                                                                                            \
        constexpr int threads = cta_threads<TPR>(), rpc = threads / TPR;                                         \
        const long long ring = Rows<T, VEC, E, TPR, 2, threads>::bytes(), cols = rpc > 1 ? rpc * 8ll * D : 0;     \
        return launch(k_norm_bwd<T, VEC, E, TPR>, grid, threads, (size_t)std::max(ring, cols), s, rows, D, x, ldx, \
                      w, mean, rstd, dy, lddy, dx, lddx, part, dw, db);                                          \
    }
    NORM_SHAPES(CALL)
    if constexpr (VEC <= 4)
        if (sh.e == 12) CALL(12, 512)
    if (sh.e == 16) CALL(16, 512)
    CALL(24, 512)  // (rows above kBwdMax take the looping kernel)
#undef CALL
}

template <class T>
cudaError_t fwd_any(const wm_seq *h, long long rows, int D, const T *x, long long ldx, const float *w, const float *b,
                    float eps, T *y, long long ldy, float *mean, float *rstd, cudaStream_t s) {
    if (D > kFwdMax) {
        const long long most = (long long)h->sms * 4;
        return launch(k_norm_fwd_long<T>, (int)(rows < most ? rows : most), kLong, 0, s, rows, D, x, ldx, w, b, eps, y, ldy, mean,
                      rstd);
    }
    constexpr int VEC = 16 / sizeof(T);
    const int v = width(VEC, sizeof(T), D, {{x, ldx}, {y, ldy}});
    if (v == VEC) return fwd<T, VEC>(h, rows, D, x, ldx, w, b, eps, y, ldy, mean, rstd, s);
    if (v == 4) return fwd<T, 4>(h, rows, D, x, ldx, w, b, eps, y, ldy, mean, rstd, s);
    if (v == 2) return fwd<T, 2>(h, rows, D, x, ldx, w, b, eps, y, ldy, mean, rstd, s);
    return fwd<T, 1>(h, rows, D, x, ldx, w, b, eps, y, ldy, mean, rstd, s);
}

template <class T>
cudaError_t bwd_any(long long rows, int D, const T *x, long long ldx, const float *w, const float *mean, const float *rstd,
                    const T *dy, long long lddy, T *dx, long long lddx, float *part, float *dw, float *db, int grid, cudaStream_t s) {
    if (D > kBwdMax)
        return launch(k_norm_bwd_long<T>, grid, kLong, 0, s, rows, D, x, ldx, w, mean, rstd, dy, lddy, dx, lddx, part);
    constexpr int VEC = 16 / sizeof(T);
    const int v = width(VEC, sizeof(T), D, {{x, ldx}, {dy, lddy}, {dx, lddx}});
    if (v == VEC) return bwd<T, VEC>(rows, D, x, ldx, w, mean, rstd, dy, lddy, dx, lddx, part, dw, db, grid, s);
    if (v == 4) return bwd<T, 4>(rows, D, x, ldx, w, mean, rstd, dy, lddy, dx, lddx, part, dw, db, grid, s);
    if (v == 2) return bwd<T, 2>(rows, D, x, ldx, w, mean, rstd, dy, lddy, dx, lddx, part, dw, db, grid, s);
    return bwd<T, 1>(rows, D, x, ldx, w, mean, rstd, dy, lddy, dx, lddx, part, dw, db, grid, s);
}

}  // namespace

cudaError_t wm_seq_norm_launch(wm_seq *h, int dtype, long long rows, int D, const void *x, long long ldx,
                               const float *w, const float *b, float eps, void *y, long long ldy, float *mean,
                               float *rstd, cudaStream_t s) {
    using bf16 = __nv_bfloat16;
    h->last_launches = 1;
    if (dtype == WM_BF16) return fwd_any(h, rows, D, (const bf16 *)x, ldx, w, b, eps, (bf16 *)y, ldy, mean, rstd, s);
    return fwd_any(h, rows, D, (const float *)x, ldx, w, b, eps, (float *)y, ldy, mean, rstd, s);
}

namespace {
int bwd_grid_of(const wm_seq *h, int dtype, long long rows, int D, const void *x, long long ldx, const void *dy, long long lddy,
                const void *dx, long long lddx) {
    return dtype == WM_BF16 ? bwd_grid<__nv_bfloat16>(h, rows, D, x, ldx, dy, lddy, dx, lddx)
                            : bwd_grid<float>(h, rows, D, x, ldx, dy, lddy, dx, lddx);
}
}  // namespace

size_t wm_seq_norm_backward_ws(const wm_seq *h, int dtype, long long rows, int D, const void *x, long long ldx, const void *dy,
                               long long lddy, const void *dx, long long lddx) {
    return (size_t)bwd_grid_of(h, dtype, rows, D, x, ldx, dy, lddy, dx, lddx) * 2 * D * sizeof(float);
}

cudaError_t wm_seq_norm_backward_launch(wm_seq *h, int dtype, long long rows, int D, const void *x, long long ldx,
                                        const float *w, const float *mean, const float *rstd, const void *dy,
                                        long long lddy, void *dx, long long lddx, float *dw, float *db,
                                        cudaStream_t s) {
    using bf16 = __nv_bfloat16;
    const int grid = bwd_grid_of(h, dtype, rows, D, x, ldx, dy, lddy, dx, lddx);
    float *part = dw || db ? (float *)h->ws : nullptr;
    h->last_launches = 0;
    if (grid > 0) {
        const cudaError_t e =
            dtype == WM_BF16
                ? bwd_any(rows, D, (const bf16 *)x, ldx, w, mean, rstd, (const bf16 *)dy, lddy, (bf16 *)dx, lddx, part, dw, db, grid, s)
                : bwd_any(rows, D, (const float *)x, ldx, w, mean, rstd, (const float *)dy, lddy, (float *)dx, lddx, part, dw, db, grid, s);
        if (e != cudaSuccess) return e;
        h->last_launches = 1;
    }
    if ((dw || db) && (grid != 1 || D > kBwdMax)) {  // no rows: zeros
        // (may start while the rows' kernel still runs: it waits for it itself)
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3((unsigned)((2 * (long long)D + 31) / 32));
        cfg.blockDim = dim3(32 * kSlices);
        cfg.stream = s;
        cudaLaunchAttribute at[1];
        at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = at;
        cfg.numAttrs = 1;
        const cudaError_t e = cudaLaunchKernelEx(&cfg, k_norm_cols, grid, D, (const float *)part, dw, db);
        if (e != cudaSuccess) return e;
        ++h->last_launches;
    }
    return cudaGetLastError();
}
