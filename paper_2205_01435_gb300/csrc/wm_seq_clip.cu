// wm_seq_clip.cu -- the global norm of many gradients, and clipping by it.
//
//   norm = sqrt(sum over all tensors of g^2);  g *= min(1, max_norm / norm)
//
// Bound by memory: every value is read for the norm, and read and written again where the
// clip applies.  The tensors go to the kernels as tables in their parameters (no copy to the
// device, no synchronisation), cut into tiles, every CTA a run of them, so that a thousand
// small tensors load the GPU as evenly as one large one and the order of the sum is fixed.
// A tile's loads are issued before the one before it is worked on.  The second launch goes
// through the runs backwards: what the first read last is still in L2.  Gradients of up to 30 MB
// take one launch, which holds them in shared memory between the norm and the clipping.
//
// Measured (one GB300): 542 MB in 60 tensors 94 us for the norm (5.8 TB/s) and 161 us for the
// clipping (6.7 TB/s); 8.8 MB in 4 tensors 10 us a call.
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

// What the gradients are multiplied by, and what the first launches leave for the second ones.
struct Scale {
    float by;    // 1: leave the gradients as they are
    float then;  // 1 but where their product is below fp32's normal range
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
__device__ __forceinline__ double squares64(const float (&v)[N]) {
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < N; ++i) s += (double)v[i] * (double)v[i];
    return s;
}

template <int N>
__device__ __forceinline__ void add_squares(const float (&v)[N], Sum &sum) {
    float s = 0.f, any = 0.f;
    if constexpr (N > 2) {  // two chains
        float r = v[1] * v[1];
        s = v[0] * v[0];
#pragma unroll
        for (int i = 2; i < N; i += 2) {
            s = fmaf(v[i], v[i], s);
            r = fmaf(v[i + 1], v[i + 1], r);
        }
        s += r;
    } else {
        s = v[0] * v[0];
    }
    // below 1e-25 squares lose bits to fp32's range, above 1e34 a sum of them could pass it
    if (s > 1e-25f && s < 1e34f) {
        sum.add(s);
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) any = fmaxf(any, fabsf(v[i]));
    if (any != 0.f || s != 0.f) sum.wide += squares64(v);  // (NaN: s is)
}

constexpr int kEach = kTileBytes / 16 / kThreads;  // 16-byte vectors of a tile per thread

// The tile that a CTA is at, and its tensor.
template <int SIZE>
struct Cursor {
    const Table<SIZE> &t;
    int i, tile;
    int lo, hi;  // the tensor's tiles
    const char *src;
    char *dst;
    long long n;
    bool bf16;
    __device__ __forceinline__ Cursor(const Table<SIZE> &table, int first) : t(table), tile(first) {
        int a = 0, b = t.count - 1;
        while (a < b) {
            const int mid = (a + b) / 2;
            if (tile < t.tile_end[mid]) b = mid;
            else a = mid + 1;
        }
        at(a);
    }
    __device__ __forceinline__ void at(int tensor) {
        i = tensor;
        lo = i ? t.tile_end[i - 1] : 0;
        hi = t.tile_end[i];
        src = (const char *)t.src[i];
        dst = (char *)t.dst[i];
        n = (long long)(t.n[i] >> 1);
        bf16 = t.n[i] & 1;
    }
    __device__ __forceinline__ void step(int by) {  // 1 or -1
        tile += by;
        if (tile >= hi && i + 1 < t.count) at(i + 1);
        else if (tile < lo && i > 0) at(i - 1);
    }
};
// A tile's place.
struct Spot {
    const char *src;
    char *dst;
    int n, vecs;  // values; 16-byte vectors among them (0: not aligned)
    bool bf16;
    template <int SIZE>
    __device__ __forceinline__ void find(const Cursor<SIZE> &c, bool with_dst) {
        bf16 = c.bf16;
        const long long at = (long long)(c.tile - c.lo) * kTileBytes;
        const int shift = bf16 ? 1 : 2;
        n = (int)min((long long)(kTileBytes >> shift), c.n - (at >> shift));
        src = c.src + at;
        dst = c.dst + at;
        vecs = (uintptr_t)src % 16 == 0 && (!with_dst || (uintptr_t)dst % 16 == 0) ? n >> (bf16 ? 3 : 2) : 0;
    }
};
// And its vectors in registers.
struct Tile : Spot {
    uint4 v[kEach];
    template <int SIZE>
    __device__ __forceinline__ void load(const Cursor<SIZE> &c, bool with_dst) {
        find(c, with_dst);
#pragma unroll
        for (int q = 0; q < kEach; ++q)
            if ((int)threadIdx.x + q * kThreads < vecs) v[q] = reinterpret_cast<const uint4 *>(src)[threadIdx.x + q * kThreads];
    }
};

// v(q): the thread's vector q of the tile.
template <class T, class F>
__device__ __forceinline__ void tile_squares(const Spot &t, F v, Sum &sum) {
    constexpr int VEC = 16 / sizeof(T);
#pragma unroll
    for (int q = 0; q < kEach; ++q)
        if ((int)threadIdx.x + q * kThreads < t.vecs) {
            const uint4 w = v(q);
            float f[VEC];
            seq_unpack(reinterpret_cast<const seq_vec<T, VEC> &>(w), f);
            add_squares(f, sum);
        }
    for (int i = t.vecs * VEC + threadIdx.x; i < t.n; i += kThreads) {
        const float f[1] = {seq_to_float(reinterpret_cast<const T *>(t.src)[i])};
        add_squares(f, sum);
    }
}
template <class F>
__device__ __forceinline__ void add_tile(const Spot &t, F v, Sum &sum) {
    if (t.bf16) tile_squares<__nv_bfloat16>(t, v, sum);
    else tile_squares<float>(t, v, sum);
}

template <class T, class F>
__device__ __forceinline__ void tile_scale(const Spot &t, F v, float scale) {
    constexpr int VEC = 16 / sizeof(T);
    T *to = reinterpret_cast<T *>(t.dst);
#pragma unroll
    for (int q = 0; q < kEach; ++q)
        if ((int)threadIdx.x + q * kThreads < t.vecs) {
            const uint4 w = v(q);
            float f[VEC];
            seq_unpack(reinterpret_cast<const seq_vec<T, VEC> &>(w), f);
#pragma unroll
            for (int k = 0; k < VEC; ++k) f[k] *= scale;
            seq_store(to + (threadIdx.x + q * kThreads) * VEC, seq_pack<T, VEC>(f));
        }
    for (int i = t.vecs * VEC + threadIdx.x; i < t.n; i += kThreads)
        to[i] = seq_from_float<T>(seq_to_float(reinterpret_cast<const T *>(t.src)[i]) * scale);
}
template <class F>
__device__ __forceinline__ void scale_tile(const Spot &t, F v, float scale) {
    if (scale == 1.f && t.src == t.dst) return;
    if (t.bf16) tile_scale<__nv_bfloat16>(t, v, scale);
    else tile_scale<float>(t, v, scale);
}

// The CTA's sum in fp64, in thread 0.
__device__ __forceinline__ double cta_sum(Sum sum, double *red) {
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
    double s = 0.0;
    if (threadIdx.x == 0)
        for (int i = 0; i < kThreads / 32; ++i) s += red[i];
    return s;
}
// The norm from the CTAs' sums, always added in the same order; in every thread.
__device__ __forceinline__ float norm_of(const double *part, int parts, double *red, float *out) {
    double s = 0.0;
    for (int i = threadIdx.x; i < parts; i += kThreads) s += __ldcg(part + i);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x / 32] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = 0.0;
        for (int i = 0; i < kThreads / 32; ++i) s += red[i];
        // (the fp64 root takes a microsecond: only where the sum is out of fp32's range)
        *out = s > 1e-30 && s < 1e38 ? sqrtf((float)s) : (float)sqrt(s);
    }
    __syncthreads();
    return *out;
}
// min(1, max_norm / norm); 1 where the norm is not finite.  A quotient below fp32's normal range has
// lost bits that values of up to 1e38 would show: it is 2^-64 times one that has not.
__device__ __forceinline__ Scale scale_of(float norm, float max_norm) {
    if (!(norm > max_norm && isfinite(norm))) return {1.f, 1.f};
    const float s = __fdiv_rn(max_norm, norm);
    return s >= 0x1p-126f ? Scale{s, 1.f} : Scale{0x1p-64f, __fdiv_rn(max_norm * 0x1p64f, norm)};
}
// Tiles [first, end) by such a product.  (Apart from the tiles' loops, where a second product, met or
// not, cost 12 registers a thread and 2% of the time of large gradients.)
template <int SIZE>
__device__ __noinline__ void scale_twice(const Table<SIZE> &t, int first, int end, Scale scale) {
    Cursor<SIZE> c(t, first);
    for (int tile = first; tile < end; ++tile, c.step(1)) {
        Spot p;
        p.find(c, true);
        for (int i = threadIdx.x; i < p.n; i += kThreads) {
            if (p.bf16)
                reinterpret_cast<__nv_bfloat16 *>(p.dst)[i] = seq_from_float<__nv_bfloat16>(
                    seq_to_float(reinterpret_cast<const __nv_bfloat16 *>(p.src)[i]) * scale.by * scale.then);
            else
                reinterpret_cast<float *>(p.dst)[i] = reinterpret_cast<const float *>(p.src)[i] * scale.by * scale.then;
        }
    }
}

// CTA b's tiles: [first, last) of an even split.
__device__ __forceinline__ int split(int tiles, int b) { return (int)((long long)tiles * b / gridDim.x); }

// part[0, parts): sums of the launches before this one and of this one's CTAs.  The last CTA of the
// last launch adds them, always in the same order, and leaves the norm and the scale.
template <int SIZE>
__global__ void __launch_bounds__(kThreads) k_clip_squares(const __grid_constant__ Table<SIZE> t, double *part, int parts_before,
                                                           int last, float max_norm, Scale *result, float *norm,
                                                           unsigned *arrived) {
    __shared__ double red[kThreads / 32];
    __shared__ float s_norm;
    __shared__ bool s_last;
    Sum sum;
    const int first = split(t.tiles, blockIdx.x), end = split(t.tiles, blockIdx.x + 1);
    Cursor<SIZE> c(t, first);
    Tile next;
    next.load(c, false);
    int vecs = 0;
    for (int tile = first; tile < end; ++tile) {
        const Tile now = next;
        if (tile + 1 < end) {
            c.step(1);
            next.load(c, false);
        }
        add_tile(now, [&](int q) { return now.v[q]; }, sum);
        if ((vecs += kTileBytes / 2 / kThreads) >= kFlush) {  // (an unaligned tile: a value a vector)
            sum.flush();
            vecs = 0;
        }
    }
    const double s = cta_sum(sum, red);
    if (threadIdx.x == 0) {
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
    const float nrm = norm_of(part, parts_before + gridDim.x, red, &s_norm);
    if (threadIdx.x == 0) {
        *norm = nrm;
        *result = scale_of(nrm, max_norm);
        *arrived = 0;
    }
}

template <int SIZE>
__global__ void __launch_bounds__(kThreads) k_clip_scale(const __grid_constant__ Table<SIZE> t, const Scale *result,
                                                         int copies) {
    const int first = split(t.tiles, blockIdx.x), end = split(t.tiles, blockIdx.x + 1);
    Cursor<SIZE> c(t, end - 1);
    // launched while the first kernel still runs: its result is there after this
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const float scale = __ldcg(&result->by), then = __ldcg(&result->then);
    if (then != 1.f) return scale_twice(t, first, end, {scale, then});
    if (scale == 1.f && !copies) return;  // (copies: some dst is not its src)
    Tile next;
    next.load(c, true);
    for (int tile = end - 1; tile >= first; --tile) {
        const Tile now = next;
        if (tile > first) {
            c.step(-1);
            next.load(c, true);
        }
        scale_tile(now, [&](int q) { return now.v[q]; }, scale);
    }
}

// ---- gradients that fit the SMs' shared memory: one launch, every value read once -----------
// All CTAs run at once (a cooperative launch), hold their tiles in shared memory, and wait for
// one another's sums.  8.8 MB took 10 us so, and 14 us in the two launches above.
constexpr int kHeld = 6;                  // tiles a CTA holds
constexpr unsigned kPolls = 1u << 20;     // the wait's limit: about a second

struct Meet {
    unsigned arrived, left;
};

template <int SIZE>
__global__ void __launch_bounds__(kThreads, 2) k_clip_once(const __grid_constant__ Table<SIZE> t, double *part, float max_norm,
                                                           float *norm, int copies, Meet *meet, int *status, uint32_t test_wait) {
    extern __shared__ uint4 held[];  // [kHeld][kEach][kThreads]
    __shared__ double red[kThreads / 32];
    __shared__ float s_norm;
    const int first = split(t.tiles, blockIdx.x), end = split(t.tiles, blockIdx.x + 1);
    auto vector = [&](int tile, int q) -> uint4 & { return held[((tile - first) * kEach + q) * kThreads + threadIdx.x]; };
    {
        Cursor<SIZE> c(t, first);
        for (int tile = first; tile < end; ++tile, c.step(1)) {
            Spot p;
            p.find(c, true);
#pragma unroll
            for (int q = 0; q < kEach; ++q)
                if ((int)threadIdx.x + q * kThreads < p.vecs)
                    copy_async<16>((uint32_t)__cvta_generic_to_shared(&vector(tile, q)), p.src + (threadIdx.x + q * kThreads) * 16);
        }
        copy_commit();
    }
    Sum sum;
    {
        Cursor<SIZE> c(t, first);
        copy_wait<0>();  // (its own copies are all that a thread reads)
        for (int tile = first; tile < end; ++tile, c.step(1)) {
            Spot p;
            p.find(c, true);
            add_tile(p, [&](int q) { return vector(tile, q); }, sum);
        }
    }
    const double s = cta_sum(sum, red);
    if (threadIdx.x == 0) {
        part[blockIdx.x] = s;
        __threadfence();
        atomicAdd(&meet->arrived, 1u);
        // (test_wait: one more than there are never arrives)
        const unsigned want = gridDim.x + (test_wait && blockIdx.x == 0), most = test_wait && blockIdx.x == 0 ? test_wait : kPolls;
        unsigned polls = 0;
        while (*(volatile unsigned *)&meet->arrived < want)
            if (++polls >= most) {
                seq_record(status + 1, WM_ERR_TIMEOUT);
                break;
            }
        __threadfence();
    }
    __syncthreads();
    const float nrm = norm_of(part, gridDim.x, red, &s_norm);
    if (threadIdx.x == 0) {
        if (blockIdx.x == 0) *norm = nrm;
        if (atomicAdd(&meet->left, 1u) == gridDim.x - 1) {  // the last to have waited: ready for the next call
            meet->arrived = 0;
            meet->left = 0;
        }
    }
    const Scale factor = scale_of(nrm, max_norm);
    if (factor.then != 1.f) return scale_twice(t, first, end, factor);
    const float scale = factor.by;
    if (scale == 1.f && !copies) return;
    Cursor<SIZE> c(t, first);
    for (int tile = first; tile < end; ++tile, c.step(1)) {
        Spot p;
        p.find(c, true);
        scale_tile(p, [&](int q) { return vector(tile, q); }, scale);
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
    Scale *result = (Scale *)h->ws;
    double *part = (double *)((char *)h->ws + 256);
    unsigned *arrived = (unsigned *)h->status + 8;
    Table<SIZE> t;
    bool copies = false;
    for (int i = 0; i < count; ++i) copies |= grads[i].n > 0 && grads[i].src != grads[i].dst;
    int left = 0;  // the last tensor that is not empty
    for (int i = 0; i < count; ++i)
        if (grads[i].n) left = i;
    if (fill(t, grads, count, 0) > left && t.tiles <= h->clip_ctas * kHeld) {
        auto *k = k_clip_once<SIZE>;
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3((unsigned)(t.tiles < h->clip_ctas ? t.tiles : h->clip_ctas));
        cfg.blockDim = dim3(kThreads);
        cfg.dynamicSmemBytes = kHeld * kTileBytes;
        cfg.stream = s;
        cudaLaunchAttribute at[1];
        at[0].id = cudaLaunchAttributeCooperative;
        at[0].val.cooperative = 1;
        cfg.attrs = at;
        cfg.numAttrs = 1;
        const uint32_t test_wait = h->test_wait;
        h->test_wait = 0;
        h->last_launches = 1;
        return cudaLaunchKernelEx(&cfg, k, (const Table<SIZE>)t, part, max_norm, norm, (int)copies, (Meet *)(h->status + 16), h->status,
                                  test_wait);
    }
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
        const cudaError_t e = cudaLaunchKernelEx(&cfg, k_clip_scale<SIZE>, (const Table<SIZE>)t, (const Scale *)result, (int)copies);
        if (e != cudaSuccess) return e;
        ++h->last_launches;
    }
    return cudaGetLastError();
}

template <int SIZE>
cudaError_t prepare_once(wm_seq *h) {
    int per_sm = 0;
    cudaError_t e = cudaFuncSetAttribute(k_clip_once<SIZE>, cudaFuncAttributeMaxDynamicSharedMemorySize, kHeld * kTileBytes);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, k_clip_once<SIZE>, kThreads, kHeld * kTileBytes);
    if (e == cudaSuccess && per_sm * h->sms < h->clip_ctas) h->clip_ctas = per_sm * h->sms;
    return e;
}

}  // namespace

// The kernels' attributes, and the CTAs that run at once (at most two an SM).
cudaError_t wm_seq_clip_prepare(wm_seq *h) {
    h->clip_ctas = 2 * h->sms;
    cudaError_t e = prepare_once<16>(h);
    if (e == cudaSuccess) e = prepare_once<128>(h);
    if (e == cudaSuccess) e = prepare_once<kTable>(h);
    return e;
}

// Room for the result and the partial sums of up to 65 tables.
size_t wm_seq_clip_ws(const wm_seq *h) { return 256 + (size_t)most_ctas(h) * 65 * sizeof(double); }

cudaError_t wm_seq_clip_launch(wm_seq *h, int count, const wm_seq_grad *grads, float max_norm, float *norm,
                               cudaStream_t s) {
    h->last_launches = 0;
    int some = 0;
    for (int i = 0; i < count; ++i) some += grads[i].n > 0;
    if (!some) return cudaMemsetAsync(norm, 0, 4, s);
    if (some <= 16) return clip<16>(h, count, grads, max_norm, norm, s);
    if (some <= 128) return clip<128>(h, count, grads, max_norm, norm, s);
    return clip<kTable>(h, count, grads, max_norm, norm, s);
}
