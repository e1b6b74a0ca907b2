// wm_seq_clip.cu -- the global norm of many gradients, and clipping by it.
//
//   norm = sqrt(sum over all tensors of g^2);  g *= min(1, max_norm / norm)
//
// Bound by memory: every value is read for the norm, and read and written again where the
// clip applies.  The tensors go to the kernels as tables in their parameters (no copy to the
// device, no synchronisation), cut into tiles that CTAs take by a fixed stride, so that a
// thousand small tensors load the GPU as evenly as one large one and the order of the sum
// is fixed.  The second launch takes the tiles from the last to the first: what the first
// read last is still in L2.
//
// Squares are summed in fp32 within a 16-byte vector (4 or 8 values) and from there on
// without rounding error that matters: a thread adds the vectors' sums into an fp32 pair
// (hi + lo, the exact error of each addition kept in lo), CTAs add in fp64.  (An fp64 add per
// vector bound the kernel: GB300 has 2 fp64 lanes an SM.)  A vector whose fp32 sum leaves the
// normal range is squared again in fp64.
#include <math.h>

#include "wm_seq_internal.h"

namespace {

constexpr int kThreads = 256, kTileBytes = 16384;
constexpr int kTable = 1024;   // tensors per launch, at most
constexpr int kFlush = 256;    // vectors per fp32 pair: 32 lanes x 256 sums below 1e34 stay finite

// The tensors of a launch (SIZE of them at most: a launch copies its whole parameter).
template <int SIZE>
struct Table {
    int count, tiles;
    const void *src[SIZE];
    void *dst[SIZE];
    unsigned long long n[SIZE];  // values << 1 | bf16
    int tile_end[SIZE];          // tiles of this and the tensors before
};

// What the first launches leave for the second ones.
struct Result {
    float scale;  // 1: leave the gradients as they are
    float norm;
};

// A sum of fp32 values as hi + lo, and in fp64 what does not fit fp32.
struct Sum {
    float hi = 0.f, lo = 0.f;
    double wide = 0.0;
    __device__ __forceinline__ void add(float v) {
        const float s = hi + v, t = s - hi;
        lo += (hi - (s - t)) + (v - t);
        hi = s;
    }
    __device__ __forceinline__ void flush() {
        wide += (double)hi + (double)lo;
        hi = lo = 0.f;
    }
};

template <int N>
__device__ __noinline__ double squares64(const float (&v)[N]) {
    double s = 0.0;
    for (int i = 0; i < N; ++i) s += (double)v[i] * (double)v[i];
    return s;
}

template <int N>
__device__ __forceinline__ void add_squares(const float (&v)[N], Sum &sum) {
    float s = 0.f, any = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) s = fmaf(v[i], v[i], s);
    // below 1e-25 squares lose bits to fp32's range, above 1e34 a sum of them could pass it
    if (s > 1e-25f && s < 1e34f) {
        sum.add(s);
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) any = fmaxf(any, fabsf(v[i]));
    if (any != 0.f || s != 0.f) sum.wide += squares64(v);  // (NaN: s is)
}

template <class T>
__device__ __forceinline__ void tile_squares(const T *p, int n, Sum &sum) {
    constexpr int VEC = 16 / sizeof(T), EACH = kTileBytes / 16 / kThreads;
    int done = 0;
    if ((uintptr_t)p % 16 == 0) {
        const int vecs = n / VEC;
        seq_vec<T, VEC> v[EACH];
#pragma unroll
        for (int q = 0; q < EACH; ++q)
            if (threadIdx.x + q * kThreads < vecs) v[q] = seq_load<T, VEC>(p + (threadIdx.x + q * kThreads) * VEC);
#pragma unroll
        for (int q = 0; q < EACH; ++q)
            if (threadIdx.x + q * kThreads < vecs) {
                float f[VEC];
                seq_unpack(v[q], f);
                add_squares(f, sum);
            }
        done = vecs * VEC;
    }
    for (int i = done + threadIdx.x; i < n; i += kThreads) {
        const float f[1] = {seq_to_float(p[i])};
        add_squares(f, sum);
    }
}

template <class T>
__device__ __forceinline__ void tile_scale(const T *p, T *q, int n, float scale) {
    constexpr int VEC = 16 / sizeof(T), EACH = kTileBytes / 16 / kThreads;
    int done = 0;
    if ((uintptr_t)p % 16 == 0 && (uintptr_t)q % 16 == 0) {
        const int vecs = n / VEC;
        seq_vec<T, VEC> v[EACH];
#pragma unroll
        for (int u = 0; u < EACH; ++u)
            if (threadIdx.x + u * kThreads < vecs) v[u] = seq_load<T, VEC>(p + (threadIdx.x + u * kThreads) * VEC);
#pragma unroll
        for (int u = 0; u < EACH; ++u)
            if (threadIdx.x + u * kThreads < vecs) {
                float f[VEC];
                seq_unpack(v[u], f);
#pragma unroll
                for (int k = 0; k < VEC; ++k) f[k] *= scale;
                seq_store(q + (threadIdx.x + u * kThreads) * VEC, seq_pack<T, VEC>(f));
            }
        done = vecs * VEC;
    }
    for (int i = done + threadIdx.x; i < n; i += kThreads) q[i] = seq_from_float<T>(seq_to_float(p[i]) * scale);
}

// The tensor that holds a tile, and the tile's first value and size.
template <int SIZE>
__device__ __forceinline__ int find(const Table<SIZE> &t, int tile, long long &first, int &n, bool &bf16) {
    int lo = 0, hi = t.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (tile < t.tile_end[mid]) hi = mid;
        else lo = mid + 1;
    }
    const int start = lo ? t.tile_end[lo - 1] : 0;
    bf16 = t.n[lo] & 1;
    const long long all = (long long)(t.n[lo] >> 1), per = kTileBytes / (bf16 ? 2 : 4);
    first = (long long)(tile - start) * per;
    n = (int)min(per, all - first);
    return lo;
}

// part[0, parts): sums of the launches before this one and of this one's CTAs.  The last CTA of the
// last launch adds them, always in the same order, and leaves the norm and the scale.
template <int SIZE>
__global__ void __launch_bounds__(kThreads) k_clip_squares(const __grid_constant__ Table<SIZE> t, double *part, int parts_before,
                                                           int last, float max_norm, Result *result, float *norm,
                                                           unsigned *arrived) {
    __shared__ double red[kThreads / 32];
    __shared__ bool s_last;
    Sum sum;
    int vecs = 0;
    for (int tile = blockIdx.x; tile < t.tiles; tile += gridDim.x) {
        long long first;
        int n;
        bool bf16;
        const int i = find(t, tile, first, n, bf16);
        if (bf16) tile_squares((const __nv_bfloat16 *)t.src[i] + first, n, sum);
        else tile_squares((const float *)t.src[i] + first, n, sum);
        if ((vecs += kTileBytes / 2 / kThreads) >= kFlush) {  // (an unaligned tile: a value a vector)
            sum.flush();
            vecs = 0;
        }
    }
    // over the warp: pairs in fp32, the wide parts only where there are any
    const bool wide = __any_sync(0xffffffffu, sum.wide != 0.0);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float h = __shfl_xor_sync(0xffffffffu, sum.hi, o), l = __shfl_xor_sync(0xffffffffu, sum.lo, o);
        sum.add(h);
        sum.lo += l;
        if (wide) sum.wide += __shfl_xor_sync(0xffffffffu, sum.wide, o);
    }
    if ((threadIdx.x & 31) == 0) {
        sum.flush();
        red[threadIdx.x / 32] = sum.wide;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        double s = 0.0;
        for (int i = 0; i < kThreads / 32; ++i) s += red[i];
        part[parts_before + blockIdx.x] = s;
        s_last = false;
        if (last) {
            __threadfence();
            s_last = atomicAdd(arrived, 1u) == gridDim.x - 1;
        }
    }
    __syncthreads();
    if (!s_last) return;
    __threadfence();
    const int parts = parts_before + gridDim.x;
    double s = 0.0;
    for (int i = threadIdx.x; i < parts; i += kThreads) s += __ldcg(part + i);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x / 32] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = 0.0;
        for (int i = 0; i < kThreads / 32; ++i) s += red[i];
        s = sqrt(s);
        *norm = result->norm = (float)s;
        const bool clip = s > (double)max_norm && isfinite((float)s);
        result->scale = clip ? (float)((double)max_norm / s) : 1.f;
        *arrived = 0;
    }
}

template <int SIZE>
__global__ void __launch_bounds__(kThreads) k_clip_scale(const __grid_constant__ Table<SIZE> t, const Result *result) {
    long long first;
    int n;
    bool bf16;
    int tile = t.tiles - 1 - (int)blockIdx.x, i = find(t, tile, first, n, bf16);
    // launched while the first kernel still runs: its result is there after this
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const float scale = __ldcg(&result->scale);
    for (;;) {
        if (scale != 1.f || t.src[i] != t.dst[i]) {
            if (bf16) tile_scale((const __nv_bfloat16 *)t.src[i] + first, (__nv_bfloat16 *)t.dst[i] + first, n, scale);
            else tile_scale((const float *)t.src[i] + first, (float *)t.dst[i] + first, n, scale);
        }
        tile -= gridDim.x;
        if (tile < 0) return;
        i = find(t, tile, first, n, bf16);
    }
}

int most_ctas(const wm_seq *h) { return h->sms * 8; }

// Fills t with the tensors from `from` on; returns how many it took.
template <int SIZE>
int fill(Table<SIZE> &t, const wm_seq_grad *g, int count, int from) {
    t.count = 0;
    long long end = 0;
    int i = from;
    for (; i < count && t.count < SIZE; ++i) {
        if (g[i].n == 0) continue;
        const bool bf = g[i].dtype == WM_BF16;
        const long long per = kTileBytes / (bf ? 2 : 4), need = (g[i].n + per - 1) / per;
        if (end + need > 0x7fffffff) break;
        end += need;
        t.src[t.count] = g[i].src;
        t.dst[t.count] = g[i].dst;
        t.n[t.count] = (unsigned long long)g[i].n << 1 | (bf ? 1 : 0);
        t.tile_end[t.count++] = (int)end;
    }
    t.tiles = (int)end;
    return i - from;
}

template <int SIZE>
cudaError_t clip(wm_seq *h, int count, const wm_seq_grad *grads, float max_norm, float *norm, cudaStream_t s) {
    Result *result = (Result *)h->ws;
    double *part = (double *)((char *)h->ws + 256);
    unsigned *arrived = (unsigned *)h->status + 8;
    Table<SIZE> t;
    bool copies = false;
    for (int i = 0; i < count; ++i) copies |= grads[i].n > 0 && grads[i].src != grads[i].dst;
    int left = 0;  // the last tensor that is not empty
    for (int i = 0; i < count; ++i)
        if (grads[i].n) left = i;
    int parts = 0;
    for (int i = 0; i <= left;) {
        i += fill(t, grads, count, i);
        const int grid = t.tiles < most_ctas(h) ? t.tiles : most_ctas(h);
        k_clip_squares<SIZE><<<grid, kThreads, 0, s>>>(t, part, parts, i > left, max_norm, result, norm, arrived);
        parts += grid;
        ++h->last_launches;
    }
    if (isinf(max_norm) && !copies) return cudaGetLastError();
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    for (int i = 0; i <= left;) {
        const bool one = i == 0;
        i += fill(t, grads, count, i);
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3((unsigned)(t.tiles < most_ctas(h) ? t.tiles : most_ctas(h)));
        cfg.blockDim = dim3(kThreads);
        cfg.stream = s;
        cfg.attrs = at;
        cfg.numAttrs = one;  // later tables follow a scale launch, whose end says nothing of the norm
        const cudaError_t e = cudaLaunchKernelEx(&cfg, k_clip_scale<SIZE>, (const Table<SIZE>)t, (const Result *)result);
        if (e != cudaSuccess) return e;
        ++h->last_launches;
    }
    return cudaGetLastError();
}

}  // namespace

// Room for the result and the partial sums of up to 65 tables.
size_t wm_seq_clip_ws(const wm_seq *h) { return 256 + (size_t)most_ctas(h) * 65 * sizeof(double); }

cudaError_t wm_seq_clip_launch(wm_seq *h, int count, const wm_seq_grad *grads, float max_norm, float *norm,
                               cudaStream_t s) {
    h->last_launches = 0;
    int some = 0;
    for (int i = 0; i < count; ++i) some += grads[i].n > 0;
    if (!some) {
        h->last_launches = 1;
        return cudaMemsetAsync(norm, 0, 4, s);
    }
    if (some <= 16) return clip<16>(h, count, grads, max_norm, norm, s);
    if (some <= 128) return clip<128>(h, count, grads, max_norm, norm, s);
    return clip<kTable>(h, count, grads, max_norm, norm, s);
}
