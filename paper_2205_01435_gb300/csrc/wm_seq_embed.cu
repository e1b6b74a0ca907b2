// wm_seq_embed.cu -- embedding lookup with scaling, and the table's gradient by sorted tokens.
//
//   out[i] = scale table[tokens[i]];   dtable[v] = scale sum_{i: tokens[i] = v} dout[i]
//
// Both are bound by memory: the lookup by writing its output, the gradient by reading dout
// once and writing the table (zeros first, then the rows that tokens took).  The gradient sorts (token, position) pairs by token,
// stably, so that a row's terms are neighbours and always come in the order of their
// positions: no floating-point atomics, the same bits every time.  Up to 12,288 tokens a CTA
// the sort is one launch of one cluster, with the pairs in shared memory; more go through
// global memory.  A warp then sums a block of sorted positions over a slice of columns in
// fp32, whatever tokens they hold, so that a token that fills half of a batch costs no more
// than tokens that come once.  A run of one token that lies inside a block is written at
// once; of a run that crosses blocks each block leaves a partial row, and a third launch adds
// these in order.  The table is filled with zeros meanwhile, by the SMs that the sort leaves
// idle.  A handful of tokens takes one launch without a sort.
//
// Measured (one GB300, durations of the kernels alone): 65,536 tokens, 512 x 1024 bf16: lookup 25 us
// (5.5 TB/s), sort 21, sums 25 us (5.4 TB/s), joining runs 9; 16,384 tokens, 30,000 x 512 fp32: lookup 8,
// sort and zeros 18, sums 10, joining 8.  The gradient's calls take 53 and 31 us.
#include <algorithm>
#include <type_traits>

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
                float f[VEC];
                seq_unpack(v[u], f);
#pragma unroll
                for (int k = 0; k < VEC; ++k) f[k] = row < 0 ? 0.f : f[k] * scale;
                seq_store(out + i * D + j, seq_pack<T, VEC>(f));
            }
        }
    }
}

// ---- the sort: least significant digit first -----------------------------------------------
// Keys are tokens, V for those outside the table (they sort last and are left out).
//
// In one cluster: CTA r holds places [r * per, (r + 1) * per) of the order in its shared memory.
// A pass ranks its pairs by digit (warps over contiguous pieces, so ranks follow the places),
// gives its digit counts to every CTA, and puts every pair to its place of the next order, in
// whichever CTA that is.
constexpr int kCluster = 16, kSortThreads = 1024, kPerCta = 12288, kSortItems = kPerCta / kSortThreads;
constexpr int kMaxDigits = 256;

struct ClusterSort {
    int n, V, per, passes, bits;  // pairs of a CTA; digit width
    unsigned per_inverse;         // floor(2^32 / per) + 1: place / per is its high product, exactly, while place * per < 2^32
    const int32_t *tokens;
    int *key, *pos;
    int *status;
    char *zero;  // filled with zeros by the launch's other clusters
    unsigned long long zero_bytes;
};

// What CTA `cta` of `ctas` fills.
__device__ __forceinline__ void fill_zeros(char *p, unsigned long long bytes, unsigned cta, unsigned ctas) {
    const unsigned long long head = min(bytes, (unsigned long long)(-(uintptr_t)p & 15)), vecs = (bytes - head) / 16;
    const unsigned long long at = (unsigned long long)cta * kSortThreads + threadIdx.x, step = (unsigned long long)ctas * kSortThreads;
    const uint4 z = make_uint4(0, 0, 0, 0);
    for (unsigned long long i = at; i < vecs; i += step) reinterpret_cast<uint4 *>(p + head)[i] = z;
    if (at < head) p[at] = 0;
    if (at < bytes - head - vecs * 16) p[head + vecs * 16 + at] = 0;
}

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t peer(const void *p, uint32_t rank) {
    uint32_t at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    return at;
}

__global__ void __launch_bounds__(kSortThreads, 1) k_sort_cluster(const ClusterSort a) {
    extern __shared__ __align__(16) unsigned char smem[];
    unsigned long long *order[2] = {reinterpret_cast<unsigned long long *>(smem),
                                    reinterpret_cast<unsigned long long *>(smem) + a.per};  // pos << 32 | key
    __shared__ __align__(4) unsigned short cnt[kSortThreads / 32][kMaxDigits];  // pairs of a digit per warp, then before it
    __shared__ int all[kCluster][kMaxDigits], base[kMaxDigits], scan[8];
    const int tid = threadIdx.x, lane = tid & 31, w = tid / 32;
    const int rank = (int)cluster_rank(), ranks = (int)cluster_size();
    const int lo = rank * a.per, m = max(0, min(a.per, a.n - lo));
    const int digits = 1 << a.bits;
    // the sums may be launched now: they wait for this grid's end before they read anything
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if ((int)blockIdx.x >= ranks) return fill_zeros(a.zero, a.zero_bytes, blockIdx.x - ranks, gridDim.x - ranks);
    for (int i = tid; i < kCluster * kMaxDigits; i += kSortThreads) all[i / kMaxDigits][i % kMaxDigits] = 0;
    if ((int)gridDim.x == ranks) fill_zeros(a.zero, a.zero_bytes, rank, ranks);
    cluster_barrier();  // every CTA has started: their shared memory may be written
    // a warp's piece of the CTA's places
    const int piece = ((a.per + 31) / 32 + 31) / 32 * 32;
    for (int pass = 0; pass < a.passes; ++pass) {
        const unsigned long long *from = order[pass & 1];
        unsigned long long *to = order[(pass & 1) ^ 1];
        for (int d = lane; d < digits / 2; d += 32) reinterpret_cast<int *>(cnt[w])[d] = 0;
        __syncthreads();
        // (kSortItems + 1: a piece is rounded up to whole warps)
        unsigned long long item[kSortItems + 1];
        unsigned short before[kSortItems + 1];
        auto mine = [&](int q) { return q * 32 < piece && w * piece + q * 32 + lane < m; };
        if (pass == 0) {  // all loads in flight together
            int t[kSortItems + 1];
#pragma unroll
            for (int q = 0; q <= kSortItems; ++q) t[q] = mine(q) ? a.tokens[lo + w * piece + q * 32 + lane] : 0;
#pragma unroll
            for (int q = 0; q <= kSortItems; ++q) {
                const int k = token_row(t[q], a.V, a.status);
                item[q] = (unsigned long long)(lo + w * piece + q * 32 + lane) << 32 | (unsigned)(k < 0 ? a.V : k);
            }
        } else {
#pragma unroll
            for (int q = 0; q <= kSortItems; ++q) item[q] = mine(q) ? from[w * piece + q * 32 + lane] : 0;
        }
#pragma unroll
        for (int q = 0; q <= kSortItems; ++q) {
            if (q * 32 >= piece || w * piece + q * 32 >= m) break;  // the same for the whole warp
            const bool in = mine(q);
            const int d = in ? ((unsigned)item[q] >> (pass * a.bits)) & (digits - 1) : digits;
            const unsigned same = __match_any_sync(0xffffffffu, d);
            const int r = __popc(same & ((1u << lane) - 1));
            const int have = in ? cnt[w][d] : 0;
            before[q] = (unsigned short)(have + r);
            __syncwarp();
            if (in && r == 0) cnt[w][d] = (unsigned short)(have + __popc(same));
            __syncwarp();
        }
        __syncthreads();
        for (int d = tid; d < digits; d += kSortThreads) {
            int c[kSortThreads / 32], sum = 0;
#pragma unroll
            for (int q = 0; q < kSortThreads / 32; ++q) c[q] = cnt[q][d];
#pragma unroll
            for (int q = 0; q < kSortThreads / 32; ++q) {
                cnt[q][d] = (unsigned short)sum;
                sum += c[q];
            }
#pragma unroll 4
            for (int q = 0; q < ranks; ++q)
                asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(peer(&all[rank][d], q)), "r"(sum) : "memory");
        }
        cluster_barrier();
        // places of smaller digits, and of this digit in the CTAs before
        if (tid < kMaxDigits) {
            int v[kCluster], total = 0, mine = 0;
#pragma unroll
            for (int q = 0; q < kCluster; ++q) v[q] = all[q][tid];  // (0 past the digits and the CTAs there are)
#pragma unroll
            for (int q = 0; q < kCluster; ++q) {
                mine += q < rank ? v[q] : 0;
                total += v[q];
            }
            int s = total;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int up = __shfl_up_sync(0xffffffffu, s, o);
                if (lane >= o) s += up;
            }
            if (lane == 31) scan[w] = s;
            asm volatile("bar.sync 1, 256;" ::: "memory");
            for (int q = 0; q < w; ++q) s += scan[q];
            base[tid] = s - total + mine;
        }
        __syncthreads();
#pragma unroll
        for (int q = 0; q <= kSortItems; ++q) {
            if (!mine(q)) break;
            const int d = ((unsigned)item[q] >> (pass * a.bits)) & (digits - 1);
            const int at = base[d] + cnt[w][d] + before[q], r = __umulhi((unsigned)at, a.per_inverse);
            asm volatile("st.shared::cluster.b64 [%0], %1;" ::"r"(peer(to + (at - r * a.per), r)), "l"(item[q]) : "memory");
        }
        cluster_barrier();
    }
    const unsigned long long *done = order[a.passes & 1];
    for (int i = tid; i < m; i += kSortThreads) {
        a.key[lo + i] = (int)(unsigned)done[i];
        a.pos[lo + i] = (int)(done[i] >> 32);
    }
}

// Through global memory, 8 bits a pass.  A pass: every tile's digit counts; their exclusive
// prefix, digits first; every pair to its place.
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
constexpr int kSum = 128;

template <class T>
struct SumArgs {
    int n, V, D, block, blocks, slices;  // sorted positions a block; slices of 32 * VEC * lane_vectors columns
    const int *key, *pos;
    const T *dout;
    T *dtable;
    float scale;
    float *part;  // [blocks][2][D]: a run that came in from the block before; one that goes on
};

// Vectors of a slice per lane: narrow accesses take more of them, so that a warp's share of a row is
// 256 bytes and more.
template <class T, int VEC>
constexpr int lane_vectors() {
    return VEC * sizeof(T) >= 8 ? 1 : VEC * sizeof(T) == 4 ? 2 : 4;
}

template <int VEC>
__device__ __forceinline__ void put(float *p, const float (&v)[VEC]) {
    *reinterpret_cast<seq_vec<float, VEC> *>(p) = *reinterpret_cast<const seq_vec<float, VEC> *>(v);
}
template <class T, int VEC>
__device__ __forceinline__ void put_row(T *p, const float (&v)[VEC], float scale) {
    float f[VEC];
#pragma unroll
    for (int k = 0; k < VEC; ++k) f[k] = v[k] * scale;
    seq_store(p, seq_pack<T, VEC>(f));
}

template <class T, int VEC>
__global__ void __launch_bounds__(kSum, 6) k_embed_sum(const SumArgs<T> a) {
    const int lane = threadIdx.x & 31;
    const long long unit = (long long)blockIdx.x * (kSum / 32) + threadIdx.x / 32;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (unit >= (long long)a.blocks * a.slices) return;
    constexpr int R = lane_vectors<T, VEC>(), U = 8 / R < 4 ? 4 : 8 / R;  // vectors of a row per lane; rows in flight
    const int b = (int)(unit / a.slices), j0 = ((int)(unit % a.slices) * 32 * R + lane) * VEC;  // columns j0 + r * 32 * VEC
    const int lo = b * a.block, hi = min(a.n, lo + a.block);
    auto mine = [&](int r) { return j0 + r * 32 * VEC < a.D; };
    // the key before the block, and whether the current run is the block's first
    const int prev = lo > 0 ? a.key[lo - 1] : -1;
    bool head = true;
    float acc[R][VEC] = {};
    // 32 keys at a time, and the one after the block (-1: after the last)
    auto key_at = [&](int i) { return i <= hi && i < a.n ? a.key[i] : -1; };
    auto pos_at = [&](int i) { return i < hi ? a.pos[i] : 0; };
    int key = key_at(lo + lane), pos = pos_at(lo + lane);
    for (int at = lo; at < hi; at += 32) {
        // the next 32 are here before this one's rows are summed
        const int nkey = key_at(at + 32 + lane), npos = pos_at(at + 32 + lane);
        const int in_next = __shfl_down_sync(0xffffffffu, key, 1), first_next = __shfl_sync(0xffffffffu, nkey, 0);
        const int after = lane == 31 ? first_next : in_next;
        // tokens outside the table come last of all: m positions count, and runs end (in the block) where a bit is set
        const int m = __popc(__ballot_sync(0xffffffffu, at + lane < hi && key < a.V));
        const unsigned ends = __ballot_sync(0xffffffffu, after != key || at + lane + 1 == hi);
#pragma unroll 1
        for (int q0 = 0; q0 < m; q0 += U) {
            seq_vec<T, VEC> v[U][R];
#pragma unroll
            for (int u = 0; u < U; ++u) {  // (past m: row 0, or a row that is not used)
                const int p = __shfl_sync(0xffffffffu, pos, (q0 + u) & 31);
                const T *row = a.dout + (long long)p * a.D;
#pragma unroll
                for (int r = 0; r < R; ++r) v[u][r] = seq_load<T, VEC>(row + (mine(r) ? j0 + r * 32 * VEC : 0));
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int q = q0 + u;
                if (q >= m) break;
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    float f[VEC];
                    seq_unpack(v[u][r], f);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) acc[r][e] += f[e];
                }
                if (!(ends >> q & 1)) continue;
                // the run ends here, or leaves the block
                const int k = __shfl_sync(0xffffffffu, key, q), nk = __shfl_sync(0xffffffffu, after, q);
                const bool came = head && k == prev, goes = nk == k;
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const int j = j0 + r * 32 * VEC;
                    if (mine(r)) {
                        if (came) put<VEC>(a.part + ((long long)b * 2) * a.D + j, acc[r]);
                        else if (goes) put<VEC>(a.part + ((long long)b * 2 + 1) * a.D + j, acc[r]);
                        else put_row<T, VEC>(a.dtable + (long long)k * a.D + j, acc[r], a.scale);
                    }
#pragma unroll
                    for (int e = 0; e < VEC; ++e) acc[r][e] = 0.f;
                }
                head = false;
            }
        }
        key = nkey;
        pos = npos;
    }
}

// A run that crosses blocks: the CTAs of the block where it starts add its parts, a CTA four slices of
// 128 columns.  A slice goes to a group of warps, whose warps take a stretch of the blocks each;
// the stretches are added in order.  (CTAs are numbered blocks first, along x alone: rows may have
// more slices than a grid's y holds.)
constexpr int kJoin = 256, kJoinColumns = 128, kJoinSlices = 4;

template <class T, int VEC>
__global__ void __launch_bounds__(kJoin) k_embed_join(const SumArgs<T> a) {
    constexpr int W = kJoin / 32, JV = VEC >= 4 ? 4 : 1, R = 4 / JV;  // a lane's columns: R times JV
    using F = seq_vec<float, JV>;
    __shared__ float s[W][R * JV][32];
    const unsigned starts = (unsigned)a.blocks - 1;  // blocks that a run can leave
    const int group = (int)(blockIdx.x / starts), b = (int)(blockIdx.x - group * starts), lo = b * a.block, hi = lo + a.block;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int k = a.key[hi - 1], k_next = a.key[hi], k_lo = a.key[lo], k_prev = lo > 0 ? a.key[lo - 1] : -1;
    if (k >= a.V || k_next != k || (k_lo == k && k_prev == k)) return;  // no run leaves, or it started before
    const int lane = threadIdx.x & 31, w = threadIdx.x / 32;
    // its last block: the last whose first key is k (32 blocks a look)
    int last;
    for (int q = b + 2;; q += 32) {
        const bool on = q + lane < a.blocks && a.key[(q + lane) * a.block] == k;
        const unsigned off = ~__ballot_sync(0xffffffffu, on);
        last = q - 1 + (off ? __ffs(off) - 1 : 32);
        if (off) break;
    }
    const int all = (a.D + kJoinColumns - 1) / kJoinColumns, first = group * kJoinSlices, slices = min(kJoinSlices, all - first);
    const int warps = W / slices, share = (last - b + warps - 1) / warps;  // warps a slice; blocks a warp
    const int sl = w / warps, part = w % warps, from = b + 1 + part * share, to = min(last + 1, from + share);
    const int j0 = (first + sl) * kJoinColumns + lane * JV;
    float acc[R * JV] = {};
    if (sl < slices) {
        // eight partial rows at a time: the run's first, then this warp's stretch (past its end: row 0, not added)
        const bool own = part == 0;
        const int rows = max(0, to - from) + own;
        for (int q0 = 0; q0 < rows; q0 += 8) {
            F v[8][R];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int q = q0 + u - own;
                const long long row = q0 + u >= rows ? 0 : q < 0 ? (long long)b * 2 + 1 : (from + q) * 2ll;
#pragma unroll
                for (int r = 0; r < R; ++r)
                    v[u][r] = *reinterpret_cast<const F *>(a.part + row * a.D + (j0 + r * 32 < a.D ? j0 + r * 32 : 0));
            }
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (q0 + u < rows)
#pragma unroll
                    for (int r = 0; r < R; ++r)
#pragma unroll
                        for (int e = 0; e < JV; ++e) acc[r * JV + e] += v[u][r].v[e];
        }
#pragma unroll
        for (int e = 0; e < R * JV; ++e) s[w][e][lane] = acc[e];
    }
    __syncthreads();
    if (sl >= slices || part) return;
    for (int q = 1; q < warps; ++q)
#pragma unroll
        for (int e = 0; e < R * JV; ++e) acc[e] += s[w + q][e][lane];
    T *to_row = a.dtable + (long long)k * a.D;
#pragma unroll
    for (int r = 0; r < R; ++r)
        if (j0 + r * 32 < a.D) {
            float f[JV];
#pragma unroll
            for (int e = 0; e < JV; ++e) f[e] = acc[r * JV + e];
            put_row<T, JV>(to_row + j0 + r * 32, f, a.scale);
        }
}

// ---- few tokens: no sort --------------------------------------------------------------------
// A warp takes a row of the table and a slice of its columns, and looks through all tokens for the
// row's, in order.  Up to kFew tokens this is one launch of 5 us where sorting first takes three and
// 20 us (41 us when all 256 tokens are one row's).
constexpr int kFew = 256, kFewThreads = 128;

template <class T, int VEC>
__global__ void __launch_bounds__(kFewThreads) k_embed_few(int n, int V, int D, const int32_t *__restrict__ tokens,
                                                           const T *__restrict__ dout, float scale, T *__restrict__ dtable,
                                                           int *status) {
    constexpr int R = lane_vectors<T, VEC>(), U = 8 / R;
    // marks[v % kMarks]: whether some token may be v (most rows are told to be empty by it alone)
    constexpr int kMarks = 4096;
    __shared__ int tok[kFew];
    __shared__ __align__(4) unsigned char marks[kMarks];
    const int lane = threadIdx.x & 31;
    for (int i = threadIdx.x; i < kMarks / 4; i += kFewThreads) reinterpret_cast<unsigned *>(marks)[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < kFew; i += kFewThreads) {
        const int t = i < n ? token_row(tokens[i], V, status) : -1;
        tok[i] = t;
        if (t >= 0) marks[t % kMarks] = 1;
    }
    __syncthreads();
    const int j0 = ((int)blockIdx.y * 32 * R + lane) * VEC;
    auto mine = [&](int r) { return j0 + r * 32 * VEC < D; };
    const long long step = (long long)gridDim.x * (kFewThreads / 32);
    for (long long v = (long long)blockIdx.x * (kFewThreads / 32) + threadIdx.x / 32; v < V; v += step) {
        float acc[R][VEC] = {};
        bool taken = false;
        for (int at = 0; at < n && marks[v % kMarks]; at += 32) {
            unsigned left = __ballot_sync(0xffffffffu, tok[at + lane] == v);
            taken |= left != 0;
            while (left) {
                seq_vec<T, VEC> x[U][R];
                const int count = __popc(left);
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const long long i = at + (left ? __ffs(left) - 1 : 0);  // (past the last: not added)
                    left &= left - 1;
#pragma unroll
                    for (int r = 0; r < R; ++r) x[u][r] = seq_load<T, VEC>(dout + i * D + (mine(r) ? j0 + r * 32 * VEC : 0));
                }
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (u < count)
#pragma unroll
                        for (int r = 0; r < R; ++r) {
                            float f[VEC];
                            seq_unpack(x[u][r], f);
#pragma unroll
                            for (int e = 0; e < VEC; ++e) acc[r][e] += f[e];
                        }
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (mine(r)) put_row<T, VEC>(dtable + v * D + j0 + r * 32 * VEC, acc[r], taken ? scale : 0.f);
    }
}

size_t up(size_t b) { return (b + 255) & ~(size_t)255; }

int key_bits(int V) {  // keys 0 ... V
    int bits = 1;
    while (bits < 31 && (V >> bits)) ++bits;
    return bits;
}

struct Layout {
    bool cluster;
    int tiles, block, blocks;
    size_t key[2], pos[2], count, part, total;
};
Layout layout(const wm_seq *h, long long n, int D, int cols) {  // cols: of a slice
    Layout l{};
    l.cluster = n <= (long long)h->sort_ranks * kPerCta;
    l.tiles = (int)((n + kTile - 1) / kTile);
    // Positions per block: all blocks' warps run at once (22 of 24 an SM), in blocks of 16 to 256 positions:
    // a second round of warps would run alone, short blocks leave more partial rows.
    const long long slices = (D + cols - 1) / cols, warps = h->sms * 22ll;
    const long long b = (n * slices + warps - 1) / warps;
    l.block = (int)(b < 16 ? 16 : b > 256 ? 256 : (b + 7) / 8 * 8);
    l.blocks = (int)((n + l.block - 1) / l.block);
    size_t o = 0;
    for (int i = 0; i < (l.cluster ? 1 : 2); ++i) {
        l.key[i] = o;
        o += up((size_t)n * 4);
        l.pos[i] = o;
        o += up((size_t)n * 4);
    }
    l.count = o;
    if (!l.cluster) o += up((size_t)l.tiles * kDigits * 4);
    l.part = o;
    o += up((size_t)l.blocks * 2 * D * 4);
    l.total = o;
    return l;
}

// Launches that may start while the one before still runs (they wait for it themselves).
template <class P>
cudaError_t follow(void (*k)(P), dim3 grid, int threads, cudaStream_t s, const P &p) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, k, p);
}

template <class T, int VEC>
constexpr int slice_columns() {
    return 32 * VEC * lane_vectors<T, VEC>();
}

template <class T, int VEC>
cudaError_t sums(wm_seq *h, SumArgs<T> a, cudaStream_t s) {
    a.slices = (a.D + slice_columns<T, VEC>() - 1) / slice_columns<T, VEC>();
    const long long warps = (long long)a.blocks * a.slices;
    cudaError_t e = follow(k_embed_sum<T, VEC>, (unsigned)((warps + kSum / 32 - 1) / (kSum / 32)), kSum, s, a);
    if (e != cudaSuccess) return e;
    ++h->last_launches;
    if (a.blocks > 1) {
        const unsigned groups = (unsigned)((a.D + kJoinColumns * kJoinSlices - 1) / (kJoinColumns * kJoinSlices));
        e = follow(k_embed_join<T, VEC>, groups * (unsigned)(a.blocks - 1), kJoin, s, a);
        ++h->last_launches;
    }
    return e;
}

// Calls f with the widest access, as an integral constant, that D and the addresses allow.
template <class T, class F>
auto by_width(int D, const void *p, const void *q, F f) {
    constexpr int VEC = 16 / sizeof(T);
    auto ok = [&](int v) { return D % v == 0 && (uintptr_t)p % (v * sizeof(T)) == 0 && (uintptr_t)q % (v * sizeof(T)) == 0; };
    if (ok(VEC)) return f(std::integral_constant<int, VEC>{});
    if constexpr (VEC == 8)
        if (ok(4)) return f(std::integral_constant<int, 4>{});
    if (ok(2)) return f(std::integral_constant<int, 2>{});
    return f(std::integral_constant<int, 1>{});
}

template <class T>
cudaError_t backward(wm_seq *h, SumArgs<T> a, const void *dout, void *dtable, cudaStream_t s) {
    a.dout = (const T *)dout;
    a.dtable = (T *)dtable;
    return by_width<T>(a.D, dout, dtable, [&](auto v) { return sums<T, decltype(v)::value>(h, a, s); });
}

template <class T>
SumArgs<T> sum_args(int n, int V, int D, const Layout &l, char *ws, int at, float scale) {
    SumArgs<T> a{};
    a.n = n; a.V = V; a.D = D; a.block = l.block; a.blocks = l.blocks;
    a.key = (const int *)(ws + l.key[at]); a.pos = (const int *)(ws + l.pos[at]);
    a.scale = scale; a.part = (float *)(ws + l.part);
    return a;
}

template <class T>
cudaError_t few(wm_seq *h, int n, int V, int D, const int32_t *tokens, const T *dout, float scale, T *dtable, cudaStream_t s) {
    return by_width<T>(D, dout, dtable, [&](auto v) {
        constexpr int VEC = decltype(v)::value;
        const long long need = ((long long)V + kFewThreads / 32 - 1) / (kFewThreads / 32), most = h->sms * 16ll;
        const dim3 grid((unsigned)(need < most ? need : most), (unsigned)((D + slice_columns<T, VEC>() - 1) / slice_columns<T, VEC>()));
        k_embed_few<T, VEC><<<grid, kFewThreads, 0, s>>>(n, V, D, tokens, dout, scale, dtable, h->status);
        h->last_launches = 1;
        return cudaGetLastError();
    });
}

template <class T>
void lookup(const wm_seq *h, long long n, int V, int D, const T *table, const int32_t *tokens, float scale, T *out,
            cudaStream_t s) {
    const long long need = (n + kLookup / 32 - 1) / (kLookup / 32), most = (long long)h->sms * 16;
    const unsigned grid = (unsigned)(need < most ? need : most);
    by_width<T>(D, table, out, [&](auto v) {
        k_embed<T, decltype(v)::value><<<grid, kLookup, 0, s>>>(n, V, D, table, tokens, scale, out, h->status);
        return 0;
    });
}

int columns(int dtype, int D, const void *dout, const void *dtable) {
    if (dtype == WM_BF16)
        return by_width<__nv_bfloat16>(D, dout, dtable, [](auto v) { return slice_columns<__nv_bfloat16, decltype(v)::value>(); });
    return by_width<float>(D, dout, dtable, [](auto v) { return slice_columns<float, decltype(v)::value>(); });
}

cudaLaunchConfig_t sort_config(int ranks, size_t smem, cudaLaunchAttribute *attr) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)ranks);
    cfg.blockDim = dim3(kSortThreads);
    cfg.dynamicSmemBytes = smem;
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)ranks;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cfg;
}

}  // namespace

// The kernel's attributes, and the largest cluster that the device takes (it has to find the SMs in
// one of its GPCs).
cudaError_t wm_seq_embed_prepare(wm_seq *h) {
    cudaError_t e = cudaFuncSetAttribute(k_sort_cluster, cudaFuncAttributeMaxDynamicSharedMemorySize, kPerCta * 16);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k_sort_cluster, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    for (h->sort_ranks = kCluster; e == cudaSuccess && h->sort_ranks > 1; h->sort_ranks /= 2) {
        cudaLaunchAttribute attr[1];
        const cudaLaunchConfig_t cfg = sort_config(h->sort_ranks, kPerCta * 16, attr);
        int clusters = 0;
        e = cudaOccupancyMaxActiveClusters(&clusters, k_sort_cluster, &cfg);
        if (e == cudaSuccess && clusters > 0) break;
    }
    return e;
}

cudaError_t wm_seq_embed_launch(wm_seq *h, int dtype, long long n, int V, int D, const void *table,
                                const int32_t *tokens, float scale, void *out, cudaStream_t s) {
    if (dtype == WM_BF16)
        lookup(h, n, V, D, (const __nv_bfloat16 *)table, tokens, scale, (__nv_bfloat16 *)out, s);
    else
        lookup(h, n, V, D, (const float *)table, tokens, scale, (float *)out, s);
    h->last_launches = 1;
    return cudaGetLastError();
}

size_t wm_seq_embed_backward_ws(const wm_seq *h, int dtype, long long n, int V, int D, const void *dout, const void *dtable) {
    return n > kFew || (D + 31) / 32 > 65535 ? layout(h, n, D, columns(dtype, D, dout, dtable)).total : 0;
}

cudaError_t wm_seq_embed_backward_launch(wm_seq *h, int dtype, long long n, int V, int D, const int32_t *tokens,
                                         const void *dout, float scale, void *dtable, cudaStream_t s) {
    const size_t es = dtype == WM_BF16 ? 2 : 4;
    h->last_launches = 0;
    if (n == 0) return cudaMemsetAsync(dtable, 0, (size_t)V * D * es, s);
    if (n <= kFew && (D + 31) / 32 <= 65535) {
        if (dtype == WM_BF16)
            return few(h, (int)n, V, D, tokens, (const __nv_bfloat16 *)dout, scale, (__nv_bfloat16 *)dtable, s);
        return few(h, (int)n, V, D, tokens, (const float *)dout, scale, (float *)dtable, s);
    }
    const Layout l = layout(h, n, D, columns(dtype, D, dout, dtable));
    char *ws = (char *)h->ws;
    const int bits = key_bits(V);
    int at = 0;
    if (l.cluster) {
        ClusterSort a{};
        a.n = (int)n; a.V = V;
        // CTAs: 1024 tokens each, as far as the cluster goes
        int ranks = 1;
        while (ranks < h->sort_ranks && (long long)ranks * kSortThreads < n) ranks *= 2;
        a.per = (int)((n + ranks - 1) / ranks);
        a.per = a.per < 2 ? 2 : a.per;
        a.per_inverse = (unsigned)((1ull << 32) / a.per + 1);
        a.passes = (bits + 7) / 8;
        a.bits = (bits + a.passes - 1) / a.passes;
        a.tokens = tokens;
        a.key = (int *)(ws + l.key[0]); a.pos = (int *)(ws + l.pos[0]);
        a.status = h->status;
        a.zero = (char *)dtable;
        a.zero_bytes = (unsigned long long)V * D * es;
        cudaLaunchAttribute attr[1];
        cudaLaunchConfig_t cfg = sort_config(ranks, (size_t)a.per * 16, attr);
        // clusters that fill, a CTA for every 64 KB as far as the SMs go; a small table the sorting one fills
        const unsigned long long ctas = std::min((a.zero_bytes >> 16) + 1, (unsigned long long)(h->sms - ranks));
        if (a.zero_bytes > (unsigned long long)ranks << 17) cfg.gridDim = dim3((unsigned)(ranks + (ctas + ranks - 1) / ranks * ranks));
        cfg.stream = s;
        const cudaError_t e = cudaLaunchKernelEx(&cfg, k_sort_cluster, a);
        if (e != cudaSuccess) return e;
        h->last_launches = 1;
    } else {
        const cudaError_t e = cudaMemsetAsync(dtable, 0, (size_t)V * D * es, s);
        if (e != cudaSuccess) return e;
        const int np = (bits + 7) / 8;
        for (int p = 0; p < np; ++p) {
            SortPass a{};
            a.n = (int)n; a.V = V; a.shift = 8 * p; a.tiles = l.tiles;
            a.tokens = p == 0 ? tokens : nullptr;
            a.key_in = (const int *)(ws + l.key[at]); a.pos_in = (const int *)(ws + l.pos[at]);
            at ^= p > 0;
            a.key_out = (int *)(ws + l.key[at]); a.pos_out = (int *)(ws + l.pos[at]);
            a.count = (int *)(ws + l.count);
            a.status = h->status;
            k_sort_count<<<l.tiles, kSort, 0, s>>>(a);
            k_sort_prefix<<<1, 1024, 0, s>>>(l.tiles * kDigits, a.count);
            k_sort_scatter<<<l.tiles, kSort, 0, s>>>(a);
            h->last_launches += 3;
        }
    }
    if (dtype == WM_BF16)
        return backward(h, sum_args<__nv_bfloat16>((int)n, V, D, l, ws, at, scale), dout, dtable, s);
    return backward(h, sum_args<float>((int)n, V, D, l, ws, at, scale), dout, dtable, s);
}
