// wm_seq_clip.cu -- the global norm of many gradients, and clipping by it.
//
//   norm = sqrt(sum over all tensors of g^2);  g *= min(1, max_norm / norm)
//
// Bound by memory: every value is read for the norm, and read and written again where the
// clip applies.  The tensors go to the kernels as tables in their parameters (no copy to the
// device, no synchronisation), cut into tiles that CTAs take by a fixed stride, so that a
// thousand small tensors load the GPU as evenly as one large one and the order of the sum
// is fixed.  Squares are fp32 within a 16-byte vector and fp64 across vectors (one fp64 add
// per 4 or 8 values stays below the fp64 rate); a vector whose fp32 sum leaves the normal
// range is squared again in fp64.
#include <math.h>

#include "wm_seq_internal.h"

namespace {

constexpr int kThreads = 256, kTileBytes = 16384;
constexpr int kTable = 1024;  // tensors per launch

struct Table {
    int count;
    const void *src[kTable];
    void *dst[kTable];
    unsigned long long n[kTable];  // values << 1 | bf16
    int tile_end[kTable];          // tiles of this and the tensors before
};

__device__ __forceinline__ double squares64(const float *v, int n) {
    double s = 0.0;
    for (int i = 0; i < n; ++i) s += (double)v[i] * (double)v[i];
    return s;
}

// The sum of squares of n <= 8 values.
template <int N>
__device__ __forceinline__ double squares(const float (&v)[N]) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) s = fmaf(v[i], v[i], s);
    // below 1e-25 the squares lose bits to fp32's range (a sum of 0 may be all zeros), above 1e37 they pass it
    if (s > 1e-25f && s < 1e37f) return (double)s;
    return squares64(v, N);
}

template <class T>
__device__ __forceinline__ double tile_squares(const T *p, long long n) {
    constexpr int VEC = 16 / sizeof(T);
    double s = 0.0;
    if ((uintptr_t)p % 16 == 0) {
        const long long vecs = n / VEC;
#pragma unroll 4
        for (long long i = threadIdx.x; i < vecs; i += kThreads) {
            const seq_vec<T, VEC> v = seq_load<T, VEC>(p + i * VEC);
            float f[VEC];
#pragma unroll
            for (int k = 0; k < VEC; ++k) f[k] = seq_to_float(v.v[k]);
            s += squares(f);
        }
        p += vecs * VEC;
        n -= vecs * VEC;
    }
    for (long long i = threadIdx.x; i < n; i += kThreads) {
        const float f[1] = {seq_to_float(p[i])};
        s += squares(f);
    }
    return s;
}

template <class T>
__device__ __forceinline__ void tile_scale(const T *p, T *q, long long n, float scale) {
    constexpr int VEC = 16 / sizeof(T);
    if ((uintptr_t)p % 16 == 0 && (uintptr_t)q % 16 == 0) {
        const long long vecs = n / VEC;
#pragma unroll 4
        for (long long i = threadIdx.x; i < vecs; i += kThreads) {
            seq_vec<T, VEC> v = seq_load<T, VEC>(p + i * VEC);
#pragma unroll
            for (int k = 0; k < VEC; ++k) v.v[k] = seq_from_float<T>(seq_to_float(v.v[k]) * scale);
            seq_store(q + i * VEC, v);
        }
        p += vecs * VEC;
        q += vecs * VEC;
        n -= vecs * VEC;
    }
    for (long long i = threadIdx.x; i < n; i += kThreads) q[i] = seq_from_float<T>(seq_to_float(p[i]) * scale);
}

// The tensor that holds a tile, and the tile's first value and size.
__device__ __forceinline__ int find(const Table &t, int tile, long long &first, long long &n, bool &bf16) {
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
    n = min(per, all - first);
    return lo;
}

__device__ __forceinline__ double cta_sum(double v, double *red) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x / 32] = v;
    __syncthreads();
    double s = red[0];
#pragma unroll
    for (int i = 1; i < kThreads / 32; ++i) s += red[i];
    return s;
}

__global__ void __launch_bounds__(kThreads) k_clip_squares(const __grid_constant__ Table t, int tiles, double *part) {
    __shared__ double red[kThreads / 32];
    double s = 0.0;
    for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        long long first, n;
        bool bf16;
        const int i = find(t, tile, first, n, bf16);
        s += bf16 ? tile_squares((const __nv_bfloat16 *)t.src[i] + first, n) : tile_squares((const float *)t.src[i] + first, n);
    }
    s = cta_sum(s, red);
    if (threadIdx.x == 0) part[blockIdx.x] = s;
}

__global__ void __launch_bounds__(kThreads) k_clip_scale(const __grid_constant__ Table t, int tiles, int parts,
                                                         const double *__restrict__ part, float max_norm, float *norm) {
    __shared__ double red[kThreads / 32];
    double s = 0.0;
    for (int i = threadIdx.x; i < parts; i += kThreads) s += part[i];
    const double nrm = sqrt(cta_sum(s, red));
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)nrm;
    const bool clip = nrm > (double)max_norm && isfinite((float)nrm);
    const float scale = clip ? (float)((double)max_norm / nrm) : 1.f;
    for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        long long first, n;
        bool bf16;
        const int i = find(t, tile, first, n, bf16);
        if (!clip && t.src[i] == t.dst[i]) continue;
        if (bf16) tile_scale((const __nv_bfloat16 *)t.src[i] + first, (__nv_bfloat16 *)t.dst[i] + first, n, scale);
        else tile_scale((const float *)t.src[i] + first, (float *)t.dst[i] + first, n, scale);
    }
}

int most_ctas(const wm_seq *h) { return h->sms * 8; }

// Fills t with the tensors from `from` on; returns how many it took and their tiles.
int fill(Table &t, const wm_seq_grad *g, int count, int from, int *tiles) {
    t.count = 0;
    long long end = 0;
    int i = from;
    for (; i < count && t.count < kTable; ++i) {
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
    *tiles = (int)end;
    return i - from;
}

}  // namespace

// Room for the partial sums of up to 64 tables.
constexpr int kTables = 64;
size_t wm_seq_clip_ws(const wm_seq *h) { return (size_t)most_ctas(h) * kTables * sizeof(double); }

cudaError_t wm_seq_clip_launch(wm_seq *h, int count, const wm_seq_grad *grads, float max_norm, float *norm,
                               cudaStream_t s) {
    h->last_launches = 0;
    double *part = (double *)h->ws;
    Table t;
    int parts = 0;
    for (int i = 0; i < count;) {
        int tiles;
        i += fill(t, grads, count, i, &tiles);
        if (!tiles) continue;
        const int grid = tiles < most_ctas(h) ? tiles : most_ctas(h);
        k_clip_squares<<<grid, kThreads, 0, s>>>(t, tiles, part + parts);
        parts += grid;
        ++h->last_launches;
    }
    bool first = true;
    for (int i = 0; i < count;) {
        int tiles;
        i += fill(t, grads, count, i, &tiles);
        if (!tiles) continue;
        const int grid = tiles < most_ctas(h) ? tiles : most_ctas(h);
        k_clip_scale<<<grid, kThreads, 0, s>>>(t, tiles, parts, part, max_norm, first ? norm : nullptr);
        first = false;
        ++h->last_launches;
    }
    if (first) {
        ++h->last_launches;
        const cudaError_t e = cudaMemsetAsync(norm, 0, 4, s);
        if (e != cudaSuccess) return e;
    }
    return cudaGetLastError();
}
