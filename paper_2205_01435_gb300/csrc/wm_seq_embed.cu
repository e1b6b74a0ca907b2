// wm_seq_embed.cu -- embedding lookup with scaling, and the table's gradient by sorted tokens.
//
//   out[i] = scale table[tokens[i]];   dtable[v] = scale sum_{i: tokens[i] = v} dout[i]
//
// Both are bound by memory: the lookup by writing its output, the gradient by reading dout
// once and writing the table once.  The gradient sorts (token, position) pairs by token,
// stably, so that a row's terms are neighbours and always come in the order of their
// positions: no floating-point atomics, the same bits every time.  A warp then sums BLOCK
// sorted positions over a slice of columns in fp32, whatever tokens they hold, so that a
// token that fills half of a batch costs no more than tokens that come once.  A run of one
// token that lies inside a block is written at once; of a run that crosses blocks each block
// leaves a partial row, and a second launch adds these in order.  Rows that no token took
// are found by binary search in the sorted tokens and filled with zeros.
#include "wm_seq_internal.h"

namespace {

__device__ __forceinline__ int token_row(int t, int V, int *status) {
    if (t >= V) seq_record(status, WM_ERR_INVALID_ARG);
    return t < 0 || t >= V ? -1 : t;
}

// ---- lookup: a warp per output row ---------------------------------------------------
constexpr int kLookup = 128;

template <class T, int VEC>
__global__ void __launch_bounds__(kLookup) k_embed(long long n, int V, int D, const T *__restrict__ table,
                                                   const int32_t *__restrict__ tokens, float scale, T *__restrict__ out,
                                                   int *status) {
    constexpr int U = 4;
    const int lane = threadIdx.x & 31;
    const long long step = (long long)gridDim.x * (kLookup / 32);
    for (long long i = (long long)blockIdx.x * (kLookup / 32) + threadIdx.x / 32; i < n; i += step) {
        const int row = token_row(tokens[i], V, status);
        const T *src = table + (long long)(row < 0 ? 0 : row) * D;
        for (int j0 = lane * VEC; j0 < D; j0 += 32 * VEC * U) {
            seq_vec<T, VEC> v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int j = j0 + u * 32 * VEC;
                if (j < D && row >= 0) v[u] = seq_load<T, VEC>(src + j);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int j = j0 + u * 32 * VEC;
                if (j >= D) break;
#pragma unroll
                for (int k = 0; k < VEC; ++k)
                    v[u].v[k] = seq_from_float<T>(row < 0 ? 0.f : seq_to_float(v[u].v[k]) * scale);
                seq_store(out + i * D + j, v[u]);
            }
        }
    }
}

// ---- the sort: least significant digit first, 8 bits a pass -----------------------------
// A pass: every tile's digit counts; their exclusive prefix, digits first; every pair to its
// place.  Keys are tokens, V for those outside the table (they sort last and are left out).
constexpr int kTile = 4096, kSort = 256, kDigits = 256;

struct SortPass {
    int n, V, shift, tiles;
    const int32_t *tokens;  // first pass: the tokens; else null
    const int *key_in, *pos_in;
    int *key_out, *pos_out;
    int *count;  // [kDigits][tiles]
    int *status;
};

__device__ __forceinline__ int sort_key(const SortPass &a, int i) {
    if (!a.tokens) return a.key_in[i];
    const int t = token_row(a.tokens[i], a.V, a.status);
    return t < 0 ? a.V : t;
}

__global__ void __launch_bounds__(kSort) k_sort_count(const SortPass a) {
    __shared__ int cnt[kDigits];
    cnt[threadIdx.x] = 0;
    __syncthreads();
    const int lo = blockIdx.x * kTile;
    for (int q = threadIdx.x; q < kTile && lo + q < a.n; q += kSort)
        atomicAdd(&cnt[(sort_key(a, lo + q) >> a.shift) & (kDigits - 1)], 1);
    __syncthreads();
    a.count[threadIdx.x * a.tiles + blockIdx.x] = cnt[threadIdx.x];
}

// Exclusive prefix sum over m counts, in place, one CTA.
__global__ void __launch_bounds__(1024) k_sort_prefix(int m, int *count) {
    __shared__ int warp_sum[32];
    int carry = 0;
    for (int base = 0; base < m; base += 1024) {
        const int i = base + threadIdx.x, lane = threadIdx.x & 31, w = threadIdx.x / 32;
        const int v = i < m ? count[i] : 0;
        int s = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int up = __shfl_up_sync(0xffffffffu, s, o);
            if (lane >= o) s += up;
        }
        if (lane == 31) warp_sum[w] = s;
        __syncthreads();
        int before = 0, total = 0;
        for (int k = 0; k < 32; ++k) {
            if (k < w) before += warp_sum[k];
            total += warp_sum[k];
        }
        if (i < m) count[i] = carry + before + s - v;
        carry += total;
        __syncthreads();
    }
}

__global__ void __launch_bounds__(kSort) k_sort_scatter(const SortPass a) {
    constexpr int W = kSort / 32;
    __shared__ int base[kDigits];       // where the next pair of each digit goes
    __shared__ int cnt[W][kDigits];     // pairs of each digit per warp, then their places
    const int lane = threadIdx.x & 31, w = threadIdx.x / 32;
    base[threadIdx.x] = a.count[threadIdx.x * a.tiles + blockIdx.x];
    const int lo = blockIdx.x * kTile, hi = min(a.n, lo + kTile);
    for (int r = lo; r < hi; r += kSort) {
        for (int q = 0; q < W; ++q) cnt[q][threadIdx.x] = 0;
        __syncthreads();
        const int i = r + threadIdx.x;
        const bool in = i < hi;
        const int key = in ? sort_key(a, i) : 0;
        const int d = in ? (key >> a.shift) & (kDigits - 1) : kDigits;
        const unsigned same = __match_any_sync(0xffffffffu, d);
        const int rank = __popc(same & ((1u << lane) - 1));
        if (in && rank == 0) cnt[w][d] = __popc(same);
        __syncthreads();
        int at = base[threadIdx.x];
        for (int q = 0; q < W; ++q) {
            const int c = cnt[q][threadIdx.x];
            cnt[q][threadIdx.x] = at;
            at += c;
        }
        base[threadIdx.x] = at;
        __syncthreads();
        if (in) {
            const int to = cnt[w][d] + rank;
            a.key_out[to] = key;
            a.pos_out[to] = a.tokens ? i : a.pos_in[i];
        }
        __syncthreads();
    }
}

// ---- sums over the sorted positions -------------------------------------------------------
constexpr int kBlock = 32, kSum = 128;

template <class T>
struct SumArgs {
    int n, V, D, blocks, slices;  // slices of 32 * VEC columns
    long long zero_warps;         // warps that look for absent rows (32 rows each)
    const int *key, *pos;
    const T *dout;
    T *dtable;
    float scale;
    float *part;  // [blocks][2][D]: a run that came in from the block before; one that goes on
};

template <class T, int VEC>
__device__ __forceinline__ void put(float *p, const float (&v)[VEC]) {
#pragma unroll
    for (int k = 0; k < VEC; ++k) p[k] = v[k];
}
template <class T, int VEC>
__device__ __forceinline__ void put_row(T *p, const float (&v)[VEC], float scale) {
    seq_vec<T, VEC> o;
#pragma unroll
    for (int k = 0; k < VEC; ++k) o.v[k] = seq_from_float<T>(v[k] * scale);
    seq_store(p, o);
}

template <class T, int VEC>
__global__ void __launch_bounds__(kSum) k_embed_sum(const SumArgs<T> a) {
    const int lane = threadIdx.x & 31;
    long long unit = (long long)blockIdx.x * (kSum / 32) + threadIdx.x / 32;
    const long long units = (long long)a.blocks * a.slices;
    if (unit >= units) {  // rows without tokens
        unit -= units;
        if (unit >= a.zero_warps) return;
        const int v = (int)unit * 32 + lane;
        int lo = 0, hi = a.n;
        while (lo < hi) {
            const int mid = lo + (hi - lo) / 2;
            if (a.key[mid] < v) lo = mid + 1;
            else hi = mid;
        }
        unsigned absent = __ballot_sync(0xffffffffu, v < a.V && (lo == a.n || a.key[lo] != v));
        float zero[VEC] = {};
        for (; absent; absent &= absent - 1) {
            const long long row = unit * 32 + __ffs(absent) - 1;
            for (int j = lane * VEC; j < a.D; j += 32 * VEC) put_row<T, VEC>(a.dtable + row * a.D + j, zero, 1.f);
        }
        return;
    }
    const int b = (int)(unit / a.slices), j = ((int)(unit % a.slices) * 32 + lane) * VEC;
    const int lo = b * kBlock, m = min(kBlock, a.n - lo);
    const int key = lane < m ? a.key[lo + lane] : a.V, pos = lane < m ? a.pos[lo + lane] : 0;
    const int prev = lo > 0 ? a.key[lo - 1] : -1, next = lo + m < a.n ? a.key[lo + m] : -1;
    const bool mine = j < a.D;
    float acc[VEC] = {};
    constexpr int U = 8;
    bool head = true;  // the current run is the block's first
#pragma unroll 1
    for (int q0 = 0; q0 < m; q0 += U) {
        seq_vec<T, VEC> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int q = q0 + u;
            const int k = __shfl_sync(0xffffffffu, key, q & 31), p = __shfl_sync(0xffffffffu, pos, q & 31);
            if (q < m && k < a.V && mine) v[u] = seq_load<T, VEC>(a.dout + (long long)p * a.D + j);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int q = q0 + u;
            const int k = __shfl_sync(0xffffffffu, key, q & 31);
            const int after = __shfl_sync(0xffffffffu, key, (q + 1) & 31);
            if (q >= m || k >= a.V) continue;
            if (mine)
#pragma unroll
                for (int e = 0; e < VEC; ++e) acc[e] += seq_to_float(v[u].v[e]);
            const bool end = q + 1 == m;
            if (!end && after == k) continue;
            // the run ends here, or leaves the block
            if (mine) {
                const bool came = head && k == prev, goes = end && k == next;
                if (came) put<T, VEC>(a.part + ((long long)b * 2) * a.D + j, acc);
                else if (goes) put<T, VEC>(a.part + ((long long)b * 2 + 1) * a.D + j, acc);
                else put_row<T, VEC>(a.dtable + (long long)k * a.D + j, acc, a.scale);
#pragma unroll
                for (int e = 0; e < VEC; ++e) acc[e] = 0.f;
            }
            head = false;
        }
    }
}

// A run that crosses blocks: the CTA of the block where it starts adds its parts, each warp a
// stretch of the blocks, then the stretches in order.
template <class T, int VEC>
__global__ void __launch_bounds__(256) k_embed_join(const SumArgs<T> a) {
    constexpr int W = 8;
    __shared__ float s[W][32 * VEC];
    const int b = blockIdx.x, hi = (b + 1) * kBlock;
    if (hi >= a.n) return;
    const int k = a.key[hi - 1];
    if (k >= a.V || a.key[hi] != k) return;
    const int lo = b * kBlock;
    if (a.key[lo] == k && lo > 0 && a.key[lo - 1] == k) return;  // it started in a block before
    // the end of the run
    int l = hi, r = a.n;
    while (l < r) {
        const int mid = l + (r - l) / 2;
        if (a.key[mid] <= k) l = mid + 1;
        else r = mid;
    }
    const int last = (l - 1) / kBlock;  // its last block
    const int lane = threadIdx.x & 31, w = threadIdx.x / 32;
    const int count = last - b, per = (count + W - 1) / W;  // blocks after this one
    const int from = b + 1 + w * per, to = min(last + 1, from + per);
    for (int sl = 0; sl < a.slices; ++sl) {
        const int j = (sl * 32 + lane) * VEC;
        float acc[VEC] = {};
        if (j < a.D) {
            if (w == 0)
#pragma unroll
                for (int e = 0; e < VEC; ++e) acc[e] = a.part[((long long)b * 2 + 1) * a.D + j + e];
#pragma unroll 4
            for (int q = from; q < to; ++q)
#pragma unroll
                for (int e = 0; e < VEC; ++e) acc[e] += a.part[((long long)q * 2) * a.D + j + e];
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) s[w][lane * VEC + e] = acc[e];
        __syncthreads();
        if (w == 0 && j < a.D) {
            for (int q = 1; q < W; ++q)
#pragma unroll
                for (int e = 0; e < VEC; ++e) acc[e] += s[q][lane * VEC + e];
            put_row<T, VEC>(a.dtable + (long long)k * a.D + j, acc, a.scale);
        }
        __syncthreads();
    }
}

size_t up(size_t b) { return (b + 255) & ~(size_t)255; }

int passes(int V) {
    int bits = 1;
    while (bits < 31 && (V >> bits)) ++bits;
    return (bits + 7) / 8;
}

struct Layout {
    int tiles, blocks;
    size_t key[2], pos[2], count, part, total;
};
Layout layout(long long n, int D) {
    Layout l{};
    l.tiles = (int)((n + kTile - 1) / kTile);
    l.blocks = (int)((n + kBlock - 1) / kBlock);
    size_t o = 0;
    for (int i = 0; i < 2; ++i) {
        l.key[i] = o;
        o += up((size_t)n * 4);
        l.pos[i] = o;
        o += up((size_t)n * 4);
    }
    l.count = o;
    o += up((size_t)l.tiles * kDigits * 4);
    l.part = o;
    o += up((size_t)l.blocks * 2 * D * 4);
    l.total = o;
    return l;
}

template <class T, int VEC>
void sums(wm_seq *h, SumArgs<T> a, cudaStream_t s) {
    a.slices = (a.D + 32 * VEC - 1) / (32 * VEC);
    const long long warps = (long long)a.blocks * a.slices + a.zero_warps;
    k_embed_sum<T, VEC><<<(unsigned)((warps + kSum / 32 - 1) / (kSum / 32)), kSum, 0, s>>>(a);
    ++h->last_launches;
    if (a.blocks > 1) {
        k_embed_join<T, VEC><<<a.blocks - 1, 256, 0, s>>>(a);
        ++h->last_launches;
    }
}

template <class T>
void backward(wm_seq *h, int n, int V, int D, const int *key, const int *pos, const T *dout, float scale, T *dtable,
              float *part, int blocks, cudaStream_t s) {
    SumArgs<T> a{};
    a.n = n; a.V = V; a.D = D; a.blocks = blocks;
    a.zero_warps = ((long long)V + 31) / 32;
    a.key = key; a.pos = pos; a.dout = dout; a.dtable = dtable; a.scale = scale; a.part = part;
    constexpr int VEC = 16 / sizeof(T);
    if (D % VEC == 0 && (uintptr_t)dout % 16 == 0 && (uintptr_t)dtable % 16 == 0) sums<T, VEC>(h, a, s);
    else sums<T, 1>(h, a, s);
}

template <class T>
void lookup(const wm_seq *h, long long n, int V, int D, const T *table, const int32_t *tokens, float scale, T *out,
            cudaStream_t s) {
    constexpr int VEC = 16 / sizeof(T);
    const long long need = (n + kLookup / 32 - 1) / (kLookup / 32), most = (long long)h->sms * 16;
    const unsigned grid = (unsigned)(need < most ? need : most);
    if (D % VEC == 0 && (uintptr_t)table % 16 == 0 && (uintptr_t)out % 16 == 0)
        k_embed<T, VEC><<<grid, kLookup, 0, s>>>(n, V, D, table, tokens, scale, out, h->status);
    else
        k_embed<T, 1><<<grid, kLookup, 0, s>>>(n, V, D, table, tokens, scale, out, h->status);
}

}  // namespace

cudaError_t wm_seq_embed_launch(wm_seq *h, int dtype, long long n, int V, int D, const void *table,
                                const int32_t *tokens, float scale, void *out, cudaStream_t s) {
    if (dtype == WM_BF16)
        lookup(h, n, V, D, (const __nv_bfloat16 *)table, tokens, scale, (__nv_bfloat16 *)out, s);
    else
        lookup(h, n, V, D, (const float *)table, tokens, scale, (float *)out, s);
    h->last_launches = 1;
    return cudaGetLastError();
}

size_t wm_seq_embed_backward_ws(const wm_seq *, long long n, int, int D) { return n ? layout(n, D).total : 0; }

cudaError_t wm_seq_embed_backward_launch(wm_seq *h, int dtype, long long n, int V, int D, const int32_t *tokens,
                                         const void *dout, float scale, void *dtable, cudaStream_t s) {
    h->last_launches = 0;
    const Layout l = layout(n, D);
    char *ws = (char *)h->ws;
    int *key[2], *pos[2];
    for (int i = 0; i < 2; ++i) {
        key[i] = (int *)(ws + l.key[i]);
        pos[i] = (int *)(ws + l.pos[i]);
    }
    int at = 0;
    if (n > 0) {
        const int np = passes(V);
        for (int p = 0; p < np; ++p) {
            SortPass a{};
            a.n = (int)n; a.V = V; a.shift = 8 * p; a.tiles = l.tiles;
            a.tokens = p == 0 ? tokens : nullptr;
            a.key_in = key[at]; a.pos_in = pos[at];
            at ^= p > 0;
            a.key_out = key[at]; a.pos_out = pos[at];
            a.count = (int *)(ws + l.count);
            a.status = h->status;
            k_sort_count<<<l.tiles, kSort, 0, s>>>(a);
            k_sort_prefix<<<1, 1024, 0, s>>>(l.tiles * kDigits, a.count);
            k_sort_scatter<<<l.tiles, kSort, 0, s>>>(a);
            h->last_launches += 3;
        }
    }
    if (dtype == WM_BF16)
        backward(h, (int)n, V, D, key[at], pos[at], (const __nv_bfloat16 *)dout, scale, (__nv_bfloat16 *)dtable,
                 (float *)(ws + l.part), l.blocks, s);
    else
        backward(h, (int)n, V, D, key[at], pos[at], (const float *)dout, scale, (float *)dtable, (float *)(ws + l.part), l.blocks, s);
    return cudaGetLastError();
}
