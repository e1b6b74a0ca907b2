// wm_seq_decay_tc.cu -- the decayed linear attention's passes in bf16 on the tensor cores (see wm_seq_decay.cu).
//
// Chunks of 128 tokens, one CTA a job of a head of a sequence (or of a span of it): 8 warps for heads of up to 64 values (two
// such CTAs an SM), 16 for up to 128, and one more that issues copies and products.  For each chunk
//   A = a b^T                     128 x 128, both K-major as they lie in memory
//   P = A * weights               TMEM -> registers -> TMEM as bf16, where the next product reads it
//   O2 = a Xb                     Xb: the state X as a bf16 tile
//   O1 = P c,  y = O1 + in_scale lambda^r O2
//   X = lambda^n X + (b w)^T c    X in fp32 in registers; b w as three bf16 values, all 24 bits of it, where the state leaves and anything of
//                                 the chunk can be left in it: it is as good as in fp32; else as two
// a, b and c lie as [128 tokens][64 values] panels of 128-byte rows in the 128-byte swizzle, which serve as K-major operands
// (a, b in A and O2) and as MN-major ones (c, and b transposed, where the tokens are summed over).  Rows come by asynchronous
// 16-byte copies that a padded token or value leaves as zeros: lengths, strides and either direction of time cost nothing extra.
// Queries and keys are two chunks ahead, values one.
//
// Rounded to bf16: P (each weight of a value by at most 2^-8 of itself, as the output is) and Xb (the state as the queries see
// it); A, O1, O2 and X are fp32.
//
// What bounds it: not the products (20% of the tensor cores' cycles for heads of 64, 35% for 128) nor memory, but
// the chain copies - A - P - O1 - update that a chunk walks, each link with its latency, and the workers' instructions between them
// (50% of the issue slots at 1024 x 64 x 16 x 64).  Hence two CTAs an SM where a head has up to 64 values (96 registers a thread are
// all that 18 warps can have), hand-overs after which the workers go on, and chunks of 128: fewer would leave half of the tensor
// cores' rows empty.  Times: 128 x 512 x 16 x 64 ragged forward 199 us (2.3 TB/s of the tokens that are there);
// 1024 x 64 x 16 x 64 forward 156 us (3.4 TB/s), backward 381 (2.5 TB/s); 8192 x 2 x 8 x 128 forward 90; 65,536 x 1 x 8 x 128 x 64
// with resets forward 235, backward 534.
//
// Masked places hold zeros, and zero times what is not finite is NaN (so is lambda = 0 times it, of log_decay = -inf): a chunk whose outputs or state are not finite marks its
// sequence, and the fp32 kernel, which skips what is masked, takes it again.
#include <algorithm>

#include "tc_ptx.cuh"
#include "wm_seq_decay.cuh"

#define TC_LD32(taddr, r)                                                                                                        \
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "                                                                       \
                 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];" \
                 : "=r"((r)[0]), "=r"((r)[1]), "=r"((r)[2]), "=r"((r)[3]), "=r"((r)[4]), "=r"((r)[5]), "=r"((r)[6]), "=r"((r)[7]), \
                   "=r"((r)[8]), "=r"((r)[9]), "=r"((r)[10]), "=r"((r)[11]), "=r"((r)[12]), "=r"((r)[13]), "=r"((r)[14]), "=r"((r)[15]), \
                   "=r"((r)[16]), "=r"((r)[17]), "=r"((r)[18]), "=r"((r)[19]), "=r"((r)[20]), "=r"((r)[21]), "=r"((r)[22]), "=r"((r)[23]), \
                   "=r"((r)[24]), "=r"((r)[25]), "=r"((r)[26]), "=r"((r)[27]), "=r"((r)[28]), "=r"((r)[29]), "=r"((r)[30]), "=r"((r)[31]) \
                 : "r"((uint32_t)(taddr)))

#define TC_ST8(taddr, r)                                                                                                         \
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};"                                        \
                 ::"r"((r)[0]), "r"((r)[1]), "r"((r)[2]), "r"((r)[3]), "r"((r)[4]), "r"((r)[5]), "r"((r)[6]), "r"((r)[7]),         \
                   "r"((uint32_t)(taddr)) : "memory")

namespace {

using bf16 = __nv_bfloat16;

constexpr int kChunk = kDecayTcChunk, kPanel = kChunk * 128;  // bytes of 128 tokens x 64 values
constexpr uint32_t kWait = 1u << 22;                                // polls of a wait (each about 20 ns or more)

// What a CTA of head width D (64 or 128) holds: shared memory and TMEM columns.
template <int D>
struct Plan {
    static constexpr int workers = 4 * D, threads = workers + 32;  // 32 columns of the state and of the outputs a thread
    static constexpr int tile = kPanel * (D / 64);
    // (lo lies behind b: with D = 64 both are one operand of 128 rows; xb's place is a tile, for the third part;
    // both also hold the state on its way in and out)
    static constexpr int b = 0, lo = b + 2 * tile, xb = lo + tile, a = xb + tile, c = a + 2 * tile, end = c + tile;
    static constexpr int small = end;  // tables and barriers
    static constexpr int notes = small + 112, bytes = notes + 128;
    // P lies over A: 16 tokens' column pairs where their warps read them, in blocks of `own` columns of A; with D = 64 O2, in two
    // halves, over the rest of each block
    static constexpr int own = 128 / (D / 32);
    static constexpr int tA = 0, tO1 = 128, tX = D == 64 ? 192 : 384, columns = D == 64 ? 256 : 512;
    static constexpr int p_at(int k) { return tA + k * 16 / own * own + k * 16 % own / 2; }     // of tokens 16 k and on
    static constexpr int o2_at(int group) { return D == 64 ? 32 + 64 * group : 256 + 32 * group; }  // of 32 outputs
};

// MN-major operand, 128-byte swizzle: 64 values a row of 128 bytes; `panel` bytes to the next 64 values, 1024 to the next
// 8 of what is summed over.
__device__ __forceinline__ uint64_t desc_mn(uint32_t saddr, uint32_t panel) {
    uint64_t d = 0;
    d |= (uint64_t)((saddr >> 4) & 0x3FFFu);
    d |= (uint64_t)((panel >> 4) & 0x3FFFu) << 16;
    d |= (uint64_t)(1024u >> 4) << 32;
    d |= (uint64_t)1u << 46;
    d |= (uint64_t)2u << 61;
    return d;
}
constexpr uint32_t kAmn = 1u << 15, kBmn = 1u << 16;  // instruction descriptor: A, B are MN-major

// The same with A in TMEM: bf16 pairs, a row a lane.
__device__ __forceinline__ void mma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}
using Pair = seq_pair;
__device__ __forceinline__ Pair pair_of(uint32_t a, uint32_t b) { return seq_pair_of(__uint_as_float(a), __uint_as_float(b)); }
__device__ __forceinline__ Pair twice(float v) { return seq_pair_of(v, v); }
__device__ __forceinline__ Pair mul2(Pair a, Pair b) { return seq_mul2(a, b); }
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) { return seq_fma2(a, b, c); }
// Two bf16 values at a time.
__device__ __forceinline__ uint32_t hmul(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t hfma(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t r;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}

// 128 tokens of an array as swizzled panels, by the CTA's threads.  `at` is the first row, step the elements to the next one;
// rows outside [lo, hi) and values that are not there are zeros.
template <int D>
__device__ __forceinline__ void load_tile(uint32_t dst, const bf16 *at, long long step, int lo, int hi, int dim, int vec) {
    constexpr int per = D / 8, stride = Plan<D>::workers / per;
    const int ch = threadIdx.x % per, row0 = threadIdx.x / per, left = dim - ch * 8;
    const bf16 *p = at + row0 * step + ch * 8;
    const uint32_t to = dst + (ch / 8) * kPanel + row0 * 128 + (((ch & 7) ^ (row0 & 7)) << 4);  // (stride is a multiple of 8)
#pragma unroll 1
    for (int k = 0; k < kChunk / stride; ++k) {
        const int row = row0 + k * stride;
        const bool on = row >= lo && row < hi && left > 0;
        if (vec > 1) {
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + k * stride * 128), "l"(on ? p : at + lo * step), "r"(on ? 16 : 0)
                         : "memory");
        } else {
            uint32_t v[4] = {};
            const unsigned short *u = reinterpret_cast<const unsigned short *>(p);
            if (on) {
#pragma unroll
                for (int h = 0; h < 8; ++h)
                    if (h < left) v[h / 2] |= (uint32_t)u[h] << (16 * (h & 1));
            }
            asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(to + k * stride * 128), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
        }
        p += stride * step;
    }
}

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap *map, int d, int t, int n, int h, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
                 "l"(map), "r"(d), "r"(t), "r"(n), "r"(h), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void tma_store_4d(const CUtensorMap *map, uint32_t src, int d, int t, int n, int h) {
    asm volatile("cp.async.bulk.tensor.4d.global.shared::cta.bulk_group [%0, {%1, %2, %3, %4}], [%5];" ::"l"(map), "r"(d), "r"(t), "r"(n), "r"(h),
                 "r"(src)
                 : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
__device__ __forceinline__ void tma_store_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void pair_barrier(int id) { asm volatile("bar.sync %0, 64;" ::"r"(id) : "memory"); }

// A state in shared memory: rows of D / 4 quads, turned so that 8 rows' quads of one column lie in 8 places.
template <int D>
__device__ __forceinline__ int state_at(int r, int quad) {
    return r * (D / 4) + (quad ^ (r & 7));
}
// Its quads in the workers' hands: quad k of rows row0, row0 + 16, ...; 4 or 8 of them a thread.
template <int D>
struct Quads {
    static constexpr int per = D / 4, turns = D * per / Plan<D>::workers, rows = Plan<D>::workers / per;
    const int k = threadIdx.x % per, row0 = threadIdx.x / per;
};
// A state [da, dc] from memory, zeros around.  Whole quads where rows and address allow.
template <int D>
__device__ __forceinline__ void state_in(float4 *x, const float *from, int da, int dc) {
    using Q = Quads<D>;
    const Q q;
    const bool wide = dc % 4 == 0 && (uintptr_t)from % 16 == 0;
    float4 v[Q::turns];
#pragma unroll
    for (int i = 0; i < Q::turns; ++i) {
        const int r = q.row0 + i * Q::rows, left = dc - 4 * q.k;
        const float *const at = from + r * dc + 4 * q.k;
        v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (r < da && left > 0) {
            if (wide) {
                v[i] = *reinterpret_cast<const float4 *>(at);
            } else {
                v[i].x = at[0];
                if (left > 1) v[i].y = at[1];
                if (left > 2) v[i].z = at[2];
                if (left > 3) v[i].w = at[3];
            }
        }
    }
#pragma unroll
    for (int i = 0; i < Q::turns; ++i) x[state_at<D>(q.row0 + i * Q::rows, q.k)] = v[i];
}
// And to memory (to = NULL: nowhere; empty: as zeros); true if a value is not finite.
template <int D>
__device__ __forceinline__ bool state_out(const float4 *x, float *to, int da, int dc, bool empty) {
    using Q = Quads<D>;
    const Q q;
    const bool wide = dc % 4 == 0 && (uintptr_t)to % 16 == 0;
    float odd = 0.f;
#pragma unroll
    for (int i = 0; i < Q::turns; ++i) {
        const int r = q.row0 + i * Q::rows, left = dc - 4 * q.k;
        if (r < da && left > 0) {
            float4 v = x[state_at<D>(r, q.k)];
            odd += v.x * 0.f;  // (values beyond the state's may be what they like)
            if (left > 1) odd += v.y * 0.f;
            if (left > 2) odd += v.z * 0.f;
            if (left > 3) odd += v.w * 0.f;
            if (to) {
                if (empty) v = make_float4(0.f, 0.f, 0.f, 0.f);
                float *const at = to + r * dc + 4 * q.k;
                if (wide) {
                    *reinterpret_cast<float4 *>(at) = v;
                } else {
                    at[0] = v.x;
                    if (left > 1) at[1] = v.y;
                    if (left > 2) at[2] = v.z;
                    if (left > 3) at[3] = v.w;
                }
            }
        }
    }
    return !(odd == 0.f);
}
// Are a chunk's keys taken in three parts?  Where the state leaves, unless nothing of what the chunk gives it is there by then: tokens
// after it may write nothing, so that a chunk's part, and two parts' 2^-17 of it, can be all there is.  (2^-277: of fp32's largest value
// less than its smallest.  Against two parts once 1/16 is left, both directions: 1024 x 64 x 16 x 64 510 -> 532 us, 65,536 x 1 x 8 x 128 x 64
// 687 -> 763.)
__device__ __forceinline__ bool in_three(float log_decay, int tokens_left) { return tokens_left <= 0 || (float)tokens_left * log_decay > -192.f; }

// 2^(rate n), rate = log2 lambda and not -inf, as good as 2^-22: for what is rounded to 2^-8.  (In registers: a look at a table in
// shared memory takes some 250 cycles beside the tensor cores' own.)
__device__ __forceinline__ float power_of(float rate, int n) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(rate * (float)n));
    return r;
}

// What the workers hand to the issuing warp: they arrive and go on, it waits.  (No worker arrives twice before it has waited:
// in between each waits for a product that was issued after, or, where a wait gave up, for the issuing warp's count of chunks.)
enum { kRead = 6, kScaled = 7, kWeighted = 8, kReady = 9 };
template <int D>
__device__ __forceinline__ void hand_over(int id) {
    asm volatile("bar.arrive %0, %1;" ::"r"(id), "n"(Plan<D>::threads) : "memory");
}
template <int D>
__device__ __forceinline__ void take_over(int id) {
    asm volatile("bar.sync %0, %1;" ::"r"(id), "n"(Plan<D>::threads) : "memory");
}
template <int D>
__device__ __forceinline__ void worker_barrier() {
    asm volatile("bar.sync 5, %0;" ::"n"(Plan<D>::workers) : "memory");
}

// TMA: the inputs have tensor maps; CUT: there may be resets.
template <int D, bool STATE, bool TMA, bool CUT>
__global__ void __launch_bounds__(Plan<D>::threads, D == 64 ? 2 : 1) decay_tc_kernel(const decay_pass p, const __grid_constant__ decay_maps maps) {
    using L = Plan<D>;
    constexpr bool early = TMA && !STATE && D == 128;  // A of the next chunk is formed as soon as P is read (O2 has a place of its own)
    extern __shared__ __align__(1024) unsigned char smem[];
    const uint32_t base = tc::smem_u32(smem);
    uint32_t *const cuts = reinterpret_cast<uint32_t *>(smem + L::small);    // [2][4]: tokens that begin something new
    volatile int *const late = reinterpret_cast<int *>(cuts + 8);           // a wait gave up
    uint32_t *const tmem_at = cuts + 9;
    volatile int *const passed = reinterpret_cast<int *>(cuts + 10);         // chunks of which the issuing warp took over all that is handed over
    const uint32_t bars = tc::smem_u32(cuts + 12), barA = bars, barO = bars + 8, barX = bars + 16, barV = bars + 24, barQK = bars + 32,
                   barEnd = bars + 48;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, quad = warp & 3;
    const bool worker = tid < L::workers;
    int jobs = 0, job_at[3] = {};
    for (int i = 0; i < p.jobs; ++i)
        if (!(STATE && p.job[i].spans_t)) job_at[jobs++] = i;
    const int pairs = p.N * p.H, items = pairs * jobs * p.spans;

    // A CTA takes items (a job of a head of a sequence, or of a span of it) one after the other.
    // (T is below 2^31 - 65536: tokens, and the ends of chunks and spans, are ints)
    struct Item {
        int at, job, pair, n, head, span, len, first, last, stop, chunks, rev;
        float g;
    };
    volatile int *const notes = reinterpret_cast<volatile int *>(smem + L::notes);  // [2][16]: items that the issuing warp has opened
    const auto open = [&](int at) {
        Item m{};
        m.at = at;
        if (at >= items) return m;
        m.span = at / (pairs * jobs);
        const int k = at - m.span * pairs * jobs;
        if (jobs == 3) {
            // the pass in time's order first, then the two against it side by side (they read the same arrays; all CTAs run the same
            // code at a time: 1024 x 64 x 16 x 64 backward 390 -> 381 us)
            m.pair = k < pairs ? k : (k - pairs) / 2;
            m.job = k < pairs ? 0 : 1 + (k - pairs) % 2;
        } else {
            m.pair = k / jobs;
            m.job = job_at[k - m.pair * jobs];
        }
        m.n = m.pair / p.H;
        m.head = m.pair - m.n * p.H;
        const decay_seq q = decay_open(p, p.job[m.job], m.n);
        m.rev = q.reverse;
        m.g = p.log_decay[m.head];
        m.len = (int)q.len;
        m.first = (int)(m.span * p.span_tokens);
        m.last = (int)min(p.T, m.span * p.span_tokens + p.span_tokens);
        m.stop = min(m.last, m.len);
        m.chunks = m.stop > m.first ? (m.stop - m.first + kChunk - 1) / kChunk : 0;
        return m;
    };
    // Row r of a chunk's tiles is token begin_of(c) + r; counted along the pass it is step step_of(r) of the chunk.
    const auto begin_of = [](const Item &m, int c) { return m.rev ? m.len - m.first - (c + 1) * kChunk : m.first + c * kChunk; };

    // Once a wait has given up, here or in another warp, those after it look once: the CTA walks to its end with what there is.
    // Its warps stay in step (see in_step), nothing more is issued, and what was is waited for at the end.
    const auto wait = [&](uint32_t bar, int phase) {
        bool there = true;
        for (uint32_t i = 0; !tc::mbar_try_wait(bar, (uint32_t)phase & 1u); ++i) {
            if (*late || i == kWait) {
                *late = 1;
                seq_record(p.status + 1, WM_ERR_TIMEOUT);
                there = false;
                break;
            }
        }
        tc::fence_after_sync();
        return there;
    };
    int asked_ab = 0, asked_c = 0;  // chunks whose copies the issuing warp asked for
    if (!worker) {
        if (tc::elect_one()) {
            for (int i = 0; i < 7; ++i) tc::mbar_init(bars + 8 * i, 1);
            tc::fence_mbar_init();
            *late = *passed = 0;
            notes[0] = notes[16] = -1;
        }
        __syncwarp();
        tc::fence_proxy_async_smem();
    }
    if (warp == 1) tc::tmem_alloc(tc::smem_u32(tmem_at), L::columns);
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    const uint32_t tmem = *tmem_at;

    if (!worker) {
        // ---- one thread issues the products, and the copies: keys and queries a chunk ahead, of the next item too
        struct Cursor {  // a chunk: of item `at`, the c-th of its `chunks`, from token t0
            int at, c, chunks, t0, dt, n, head, maps, left;  // left: tokens of the sequence from this chunk's end on
            float g;
            bool enters, fine;
        };
        int opened = 0;
        bool goes = true;  // no wait of this warp has given up: what it issues finds its operands, and its barriers in step
        const auto await = [&](uint32_t bar, int phase) { goes = __all_sync(~0u, wait(bar, phase)) && goes; };
        const auto find = [&](Cursor &k, int at) {  // the first chunk of item `at`, or of the next one that has any
            for (;; at += gridDim.x) {
                const Item m = open(at);
                if (TMA && m.chunks > 0) {
                    // for the workers, who are at the item before (and past the one before that, whose place this is): what opening it
                    // takes, looks at memory among it, is done when they come to it
                    if (lane == 0) {
                        volatile int *const note = notes + (opened & 1) * 16;
                        note[1] = m.job, note[2] = m.pair, note[3] = m.n, note[4] = m.head, note[5] = m.span, note[6] = m.len, note[7] = m.first;
                        note[8] = m.last, note[9] = m.stop, note[10] = m.chunks, note[11] = m.rev, note[12] = __float_as_int(m.g);
                        __threadfence_block();
                        note[0] = m.at;
                    }
                    ++opened;
                }
                const decay_job &j = p.job[m.job];
                k = {at, 0, m.chunks, begin_of(m, 0), m.rev ? -kChunk : kChunk, m.n, m.head, j.map[0] | j.map[1] << 2 | j.map[2] << 4,
                     m.len - m.first - kChunk, m.g, !STATE && (p.spans > 1 || j.s_in), j.fine != 0};
                if (m.chunks > 0 || at >= items) return;
            }
        };
        const auto step = [&](Cursor &k) {
            k.t0 += k.dt;
            k.left -= kChunk;
            if (++k.c >= k.chunks && k.at < items) find(k, k.at + (int)gridDim.x);
        };
        const auto load = [&](const Cursor &k, uint32_t dst, int map, uint32_t bar) {
#pragma unroll
            for (int i = 0; i < D / 64; ++i) tma_load_4d(dst + i * kPanel, &maps.in[map], i * 64, k.t0, k.n, k.head, bar);
        };
        const auto load_ab = [&](const Cursor &k, int slot) {  // keys, and queries
            if (k.at >= items || !goes) return;
            ++asked_ab;
            if (tc::elect_one()) {
                tc::mbar_arrive_expect_tx(barQK + 8 * slot, (STATE ? 1 : 2) * L::tile);
                load(k, base + L::b + slot * L::tile, k.maps >> 2 & 3, barQK + 8 * slot);
                if constexpr (!STATE) load(k, base + L::a + slot * L::tile, k.maps & 3, barQK + 8 * slot);
            }
            __syncwarp();
        };
        const auto load_c = [&](const Cursor &k) {
            if (k.at >= items || !goes) return;
            ++asked_c;
            if (tc::elect_one()) {
                tc::mbar_arrive_expect_tx(barV, L::tile);
                load(k, base + L::c, k.maps >> 4, barV);
            }
            __syncwarp();
        };
        Cursor now;
        find(now, blockIdx.x);
        Cursor ahead = now;
        if constexpr (TMA) {
            load_ab(ahead, 0);
            load_c(ahead);
            step(ahead);
            load_ab(ahead, 1);
        }
        const auto form_a = [&](int slot) {
            const uint32_t ta = base + L::a + slot * L::tile, tb = base + L::b + slot * L::tile;
            if (goes && tc::elect_one()) {
#pragma unroll
                for (int k = 0; k < D / 16; ++k)
                    tc::mma_bf16(tmem + L::tA, tc::desc_sw128(ta + (k / 4) * kPanel + (k % 4) * 32), tc::desc_sw128(tb + (k / 4) * kPanel + (k % 4) * 32),
                                 tc::idesc_bf16_f32(128, 128), k > 0);
                tc::mma_commit(barA);
            }
            __syncwarp();
        };
        const auto test = [&]() {  // (a test's wait, for what nothing sets)
            if (!p.test_wait || blockIdx.x != 0) return;
            if (!tc::mbar_wait_bounded(barEnd, 0, p.test_wait)) {
                *late = 1;
                seq_record(p.status + 1, WM_ERR_TIMEOUT);
            }
            goes = false;
        };
        if (now.at >= items) test();
#pragma unroll 1
        for (int done = 0; now.at < items; ++done) {  // chunks
            const bool has_x = now.enters || now.c > 0, fine = now.fine && in_three(now.g, now.left);
            const int slot = done & 1;
            const uint32_t ta = base + L::a + slot * L::tile, tb = base + L::b + slot * L::tile, tv = base + L::c;
            if (done == (TMA && ahead.at < items ? 1 : 0)) test();  // (where there is a second chunk, with copies and products on their way)
            if (TMA && !(early && done > 0)) await(barQK + 8 * slot, done >> 1);
            take_over<D>(kRead);  // the chunk before is read out
            tc::fence_after_sync();
            if (!STATE && !(early && done > 0)) form_a(slot);
            if (TMA && done > 0) {
                step(ahead);
                load_ab(ahead, slot ^ 1);
            }
            if (!STATE) {
                take_over<D>(kScaled);  // A is read, Xb there
                tc::fence_after_sync();
            }
            if (!STATE && has_x && goes && tc::elect_one()) {
                constexpr int parts = D == 64 ? 2 : 1;
#pragma unroll
                for (int part = 0; part < parts; ++part)
#pragma unroll
                    for (int k = 0; k < D / 16; ++k)
                        tc::mma_bf16(tmem + L::o2_at(part), tc::desc_sw128(ta + (k / 4) * kPanel + (k % 4) * 32),
                                     desc_mn(base + L::xb + k * 2048 + part * 64, D * 128), tc::idesc_bf16_f32(128, D / parts) | kBmn, k > 0);
            }
            __syncwarp();
            if constexpr (TMA) await(barV, done);
            if constexpr (!STATE) {
                take_over<D>(kWeighted);  // P is there
                tc::fence_after_sync();
                if (goes && tc::elect_one()) {
#pragma unroll
                    for (int k = 0; k < kChunk / 16; ++k)
                        mma_bf16_ts(tmem + L::tO1, tmem + L::p_at(k), desc_mn(tv + k * 2048, kPanel), tc::idesc_bf16_f32(128, D) | kBmn, k > 0);
                    tc::mma_commit(barO);
                }
                __syncwarp();
            }
            take_over<D>(kReady);  // the keys' parts are there
            tc::fence_after_sync();
            if (lane == 0) *passed = done + 1;
            if (goes && tc::elect_one()) {
                // (D = 64: two operands of 128 rows, the first two parts and half of the third twice)
                const auto update = [&](uint32_t at, uint32_t panel, bool more) {
#pragma unroll
                    for (int k = 0; k < kChunk / 16; ++k)
                        tc::mma_bf16(tmem + L::tX, desc_mn(at + k * 2048, panel), desc_mn(tv + k * 2048, kPanel),
                                     tc::idesc_bf16_f32(128, D) | kAmn | kBmn, more || k > 0);
                };
                // the smallest first: what the tensor cores' sums lose, by cutting them off at 24 bits, is a part of what is there
                if (fine) update(base + L::xb, D == 128 ? kPanel : 0, false);
                if (D == 128) update(base + L::lo, kPanel, fine);
                update(tb, D == 128 ? kPanel : base + L::lo - tb, fine || D == 128);
                tc::mma_commit(barX);
            }
            __syncwarp();
            if constexpr (TMA) now = ahead;
            else step(now);
            if (early && now.at < items) {
                await(barQK + 8 * (slot ^ 1), (done + 1) >> 1);
                form_a(slot ^ 1);
            }
            if (TMA) {
                await(barX, done);
                load_c(now);
            }
        }
    } else {
        const uint32_t mine = tmem + ((uint32_t)(quad * 32) << 16);
        const int xrow = quad * 32 + lane, group = warp >> 2, col0 = group * 32;
        float4 *const x = reinterpret_cast<float4 *>(smem + L::lo);  // a state on its way
        // (The products that the workers wait for are what keeps them from arriving twice at what the issuing warp has not taken over.
        // Without them its count of chunks does.  It gets there: no worker waits for it on the way but in bounded waits and here.)
        const auto in_step = [&](int phase) {
            for (uint32_t i = 0; *passed <= phase && i < (1u << 26); ++i) __nanosleep(100);
        };
        int done = 0;                                                // chunks
        int taken = 0;                                               // items that had any
        Item m = open(blockIdx.x);
        while (m.at < items) {
            const decay_job &j = p.job[m.job];
            const int da = j.da, dc = j.dc, len = m.len, first = m.first, last = m.last, stop = m.stop, chunks = m.chunks;
            const bool rev = m.rev;
            const float g = m.g;
            const decay_seq q{p.T, len, rev};
            const int cells = da * dc;
            bf16 *const py = static_cast<bf16 *>(const_cast<void *>(j.y.p)) + m.n * j.y.n + m.head * j.y.h;
            const auto step_of = [&](int r) { return rev ? kChunk - 1 - r : r; };
            const auto find_cuts = [&](int c) {
                if (CUT && warp < 4) {
                    const int s = first + c * kChunk + warp * 32 + lane;
                    const unsigned bits = __ballot_sync(~0u, c < chunks && s < stop && decay_cut(p, q, s, m.n, g));
                    if (lane == 0) cuts[((done + c) & 1) * 4 + warp] = bits;
                }
            };
            const float *from = nullptr;  // the entering state
            int from_t = 0;
            if constexpr (!STATE) {
                if (p.spans > 1) {
                    from = j.spans + ((long long)m.span * pairs + m.pair) * cells;
                    from_t = j.spans_t;
                } else if (j.s_in) {
                    from = j.s_in + (long long)m.pair * cells;
                    from_t = j.in_t;
                }
            }
            const bool enters = from != nullptr;
            bool bad = false;   // something was not finite
            bool keeps = true;  // (STATE) no cut so far
            // (without TMA the workers load: keys and queries a chunk ahead within an item)
            const auto load = [&](int c, uint32_t dst, const decay_array &g, int dim) {
                const int n = min(kChunk, stop - first - c * kChunk);
                load_tile<D>(dst, static_cast<const bf16 *>(g.p) + m.n * g.n + m.head * g.h + begin_of(m, c) * g.t, g.t, rev ? kChunk - n : 0, rev ? kChunk : n,
                             dim, j.vec);
            };
            const auto load_ab = [&](int c) {
                const int slot = (done + c) & 1;
                if (c < chunks) {
                    load(c, base + L::b + slot * L::tile, j.b, da);
                    if constexpr (!STATE) load(c, base + L::a + slot * L::tile, j.a, da);
                }
                copy_commit();
            };
            const auto load_c = [&](int c) {
                if (c < chunks) load(c, base + L::c, j.c, dc);
                copy_commit();
            };
            if constexpr (!TMA) {
                load_ab(0);
                load_c(0);
                load_ab(1);
            }
            find_cuts(0);
            const float log2_lambda = g * 1.4426950408889634f, rate = log2_lambda < -1e4f ? -1e4f : log2_lambda;  // (NaN stays NaN)
            const float w_scale = j.w_scale, in_scale = j.in_scale, up_scale = j.up_scale;
            worker_barrier<D>();
            // The state, in registers: of row xr, columns xc and on.  The products of a chunk come by TMEM, fresh each time: the tensor
            // cores' sums are cut off, not rounded, which a state that they ran on over a long sequence would feel (the state's
            // gradient after 16,384 tokens of 8 heads of 128: 2e-7 off in the norm, by sums in place in TMEM 1e-6; that is what it
            // costs, when it was built: 65,536 x 1 x 8 x 128 x 64 479 -> 547 us backward, 1024 x 64 x 16 x 64 371 -> 389).
            constexpr int XN = D == 64 ? 16 : 32;
            const int xr = D == 64 ? xrow & 63 : xrow, xc = col0 + (D == 64 && quad >= 2 ? 16 : 0);
            float X[XN];
#pragma unroll
            for (int i = 0; i < XN; ++i) X[i] = 0.f;
            if (enters && chunks > 0) {
                const float mul = p.spans == 1 && j.first ? decay_power(g, 1) : 1.f;
                if (from_t) {  // (a row of the state is a column there: lanes read side by side)
#pragma unroll
                    for (int i = 0; i < XN; ++i) X[i] = xr < da && xc + i < dc ? from[(xc + i) * da + xr] : 0.f;
                } else {
                    state_in<D>(x, from, da, dc);
                    worker_barrier<D>();
#pragma unroll
                    for (int i = 0; i < XN; i += 4) {
                        const float4 v = x[state_at<D>(xr, (xc + i) / 4)];
                        X[i] = v.x, X[i + 1] = v.y, X[i + 2] = v.z, X[i + 3] = v.w;
                    }
                    // (all have read it: with D = 128 the state lies over lo and xb, and xb is written before the workers meet again,
                    // lo after a product that may have been formed ahead; where there are cuts to find they meet at the chunk's head)
                    if constexpr (D == 128 && TMA && !CUT) worker_barrier<D>();
                }
                if (mul != 1.f) {
#pragma unroll
                    for (int i = 0; i < XN; ++i) X[i] *= mul;
                }
            }
            // X <- shrink X (keep) + the last chunk's products.  D = 64: those are the sums of lanes 0 to 63 (of the keys' first parts) and
            // 64 to 127 (of the second); two threads share a row's 32 columns and send each other what the other one adds, one by way of
            // their own places in Xb, one by the places behind it.
            const auto fold = [&](float shrink, bool keep) {
                if constexpr (D == 128) {
#pragma unroll
                    for (int h = 0; h < 32; h += 16) {
                        uint32_t r[16];
                        __syncwarp();
                        TC_LD16(mine + L::tX + col0 + h, r);
                        tc::tmem_ld_wait();
#pragma unroll
                        for (int i = 0; i < 16; ++i) X[h + i] = keep ? X[h + i] * shrink + __uint_as_float(r[i]) : __uint_as_float(r[i]);
                    }
                } else {
                    uint32_t r[32];
                    __syncwarp();
                    TC_LD32(mine + L::tX + col0, r);
                    tc::tmem_ld_wait();
                    const uint32_t row = base + L::xb + xr * 128, far = base + L::xb + 8192 + (group * 64 + xr) * 64;
                    const auto near_at = [&](int i) { return row + (((group * 4 + i / 4) ^ (xr & 7)) << 4); };
                    const auto far_at = [&](int i) { return far + (((i / 4) ^ ((xr >> 1) & 3)) << 4); };
                    const bool low = quad < 2;
                    if (low) {
#pragma unroll
                        for (int i = 0; i < 16; i += 4)
                            asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(far_at(i)), "r"(r[16 + i]), "r"(r[17 + i]), "r"(r[18 + i]), "r"(r[19 + i]) : "memory");
                    } else {
#pragma unroll
                        for (int i = 0; i < 16; i += 4)
                            asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(near_at(i)), "r"(r[i]), "r"(r[i + 1]), "r"(r[i + 2]), "r"(r[i + 3]) : "memory");
                    }
                    pair_barrier(1 + group * 2 + (quad & 1));
                    uint32_t e[16];
#pragma unroll
                    for (int i = 0; i < 16; i += 4)
                        asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(e[i]), "=r"(e[i + 1]), "=r"(e[i + 2]), "=r"(e[i + 3]) : "r"(low ? near_at(i) : far_at(i)) : "memory");
                    if (!low) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) r[i] = r[16 + i];
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) + __uint_as_float(e[i]));
                    pair_barrier(1 + group * 2 + (quad & 1));  // (both have read: Xb may take its place)
#pragma unroll
                    for (int i = 0; i < 16; ++i) X[i] = keep ? X[i] * shrink + __uint_as_float(r[i]) : __uint_as_float(r[i]);
                }
            };
            bool kept = true;    // no cut in the last chunk
            float shrink = 1.f;  // what the state keeps over it (STATE: weights are up to the span's end)
            uint32_t odd = 0;  // two bf16: NaN once an output was not finite
            const int step = step_of(xrow);

#pragma unroll 1
            for (int c = 0; c < chunks; ++c) {
                const int s0 = first + c * kChunk, t0 = begin_of(m, c), rows = min(kChunk, stop - s0), slot = (done + c) & 1, phase = done + c;
                const bool fine = j.fine && in_three(g, len - s0 - kChunk);
                const uint32_t ta = base + L::a + slot * L::tile, tb = base + L::b + slot * L::tile, tv = base + L::c;
                const bool has_x = enters || c > 0;
                if constexpr (!TMA) copy_wait<1>();
                if constexpr (!STATE) tma_store_read();  // (the outputs' copies have read a's tile, which is filled again)
                tc::fence_proxy_async_smem();
                tc::fence_before_sync();
                if (CUT || !TMA) worker_barrier<D>();  // the chunk's cuts, or its tiles, are there
                hand_over<D>(kRead);
                if (!TMA && c > 0) load_ab(c + 1);
                // tokens that begin something new: what a token sees begins with the last of them up to it (counted in steps)
                int keep_from = -1, begin = -1;
                bool any_cut = false;
                if constexpr (CUT) {
                    uint32_t cut[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) cut[i] = cuts[slot * 4 + i];
                    any_cut = (cut[0] | cut[1] | cut[2] | cut[3]) != 0;
                    if (any_cut) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            if (cut[i]) keep_from = 32 * i + 31 - __clz(cut[i]);  // (no cuts behind the last step)
                            const uint32_t m = step / 32 > i ? cut[i] : step / 32 < i ? 0u : cut[i] & (~0u >> (31 - step % 32));
                            if (m) begin = 32 * i + 31 - __clz(m);
                        }
                    }
                    if constexpr (STATE) keeps = keeps && keep_from < 0;
                }
                // (time's order, the last token of all: the state leaves as that token wrote it)
                const int less = !STATE && j.first && s0 + rows == len ? 1 : 0;
                if (STATE && TMA) wait(barQK + 8 * slot, phase >> 1);
                if (c > 0) fold(shrink, kept);
                kept = keep_from < 0;
                shrink = STATE ? 1.f : decay_power(g, rows - less);
                if (STATE && c > 0) worker_barrier<D>();  // (what they sent each other is read: the third parts take its place)
                constexpr int cols = 128 / (D / 32);  // of A, a thread
                // Is any of the warp's 32 rows there?  (Those that are not keep what A left, which reaches no row but their own.
                // 128 x 512 x 16 x 64 ragged 199 -> 193 us, 65,536 x 1 x 8 x 128 x 64 forward 196 -> 201, for its spilled registers.)
                const bool live = rev ? quad * 32 + 32 > kChunk - rows : quad * 32 < rows;
                if constexpr (!STATE) {
                    if (has_x) {  // X -> Xb
                        const uint32_t to = base + L::xb + (xc / 64) * (D * 128) + xr * 128;
#pragma unroll
                        for (int i = 0; i < XN; i += 8)
                            asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(to + ((((xc % 64 + i) / 8) ^ (xr & 7)) << 4)), "r"(pack2(X[i], X[i + 1])),
                                         "r"(pack2(X[i + 2], X[i + 3])), "r"(pack2(X[i + 4], X[i + 5])), "r"(pack2(X[i + 6], X[i + 7])) : "memory");
                    }
                    // A -> P: row xrow, 16 columns at a time, P over columns that are read.  Weights lambda^away by products from the
                    // nearest column on: up to 16 roundings of 2^-24, before one of 2^-8.  (A loop, for the instructions' cache: 1024 x 64 x 16 x 64
                    // backward 389 -> 359 us, unrolled against not; 65,536 x 1 x 8 x 128 x 64 forward 201 -> 196)
                    wait(barA, phase);
#pragma unroll 1
                    for (int h = 0; h < (live ? cols / 16 : 0); ++h) {
                        const int j0 = group * cols + h * 16, block = j0 / 32;
                        uint32_t v[16];
                        if (rev ? block < quad : block > quad) {  // not seen
#pragma unroll
                            for (int i = 0; i < 8; ++i) v[i] = 0u;
                        } else {
                            TC_LD16(mine + L::tA + j0, v);
                            const float lambda = power_of(rate, 1);
                            // (the weight of the column before the first of these, in the order they are taken)
                            const int before = rev ? j0 - 1 - xrow : xrow - j0 - 16;
                            float w = before >= 0 ? w_scale * power_of(rate, before) : 0.f;
                            const auto weigh = [&](int i, float a, float b) {
                                const Pair t = mul2(pair_of(v[i], v[i + 1]), seq_pair_of(a, b));
                                v[i] = __float_as_uint(t.f.x), v[i + 1] = __float_as_uint(t.f.y);
                            };
                            tc::tmem_ld_wait();
                            if (block == quad) {  // columns behind the token itself are not seen, whatever they hold
                                const int own = lane - j0 % 32;
                                if (!rev) {
#pragma unroll
                                    for (int i = 14; i >= 0; i -= 2) {
                                        const float b = i + 1 == own ? w_scale : w * lambda;
                                        w = i == own ? w_scale : b * lambda;
                                        v[i + 1] = i + 1 <= own ? v[i + 1] : 0u;
                                        v[i] = i <= own ? v[i] : 0u;
                                        weigh(i, w, b);
                                    }
                                } else {
#pragma unroll
                                    for (int i = 0; i < 16; i += 2) {
                                        const float a = i == own ? w_scale : w * lambda;
                                        w = i + 1 == own ? w_scale : a * lambda;
                                        v[i] = i >= own ? v[i] : 0u;
                                        v[i + 1] = i + 1 >= own ? v[i + 1] : 0u;
                                        weigh(i, a, w);
                                    }
                                }
                            } else {
                                const Pair lambda2 = twice(lambda * lambda);
                                w *= lambda;
                                Pair t = rev ? seq_pair_of(w, w * lambda) : seq_pair_of(w * lambda, w);
                                if (!rev) {
#pragma unroll
                                    for (int i = 14; i >= 0; i -= 2, t = mul2(t, lambda2)) weigh(i, t.f.x, t.f.y);
                                } else {
#pragma unroll
                                    for (int i = 0; i < 16; i += 2, t = mul2(t, lambda2)) weigh(i, t.f.x, t.f.y);
                                }
                            }
                            if (CUT && any_cut) {
#pragma unroll
                                for (int i = 0; i < 16; ++i) v[i] = step_of(j0 + i) >= begin ? v[i] : 0u;
                            }
#pragma unroll
                            for (int i = 0; i < 8; ++i) v[i] = pack2(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1]));
                        }
                        __syncwarp();
                        TC_ST8(mine + L::tA + group * cols + h * 8, v);
                    }
                }
                if constexpr (!STATE) {
                    tc::fence_proxy_async_smem();  // Xb
                    tc::fence_before_sync();
                    hand_over<D>(kScaled);
                }
                if constexpr (TMA) {
                    if (rows < kChunk) {  // values of steps that are not there: whatever lies there times 0 is to be 0
                        wait(barV, phase);
                        constexpr int per = D / 8;
                        for (int i = tid; i < (kChunk - rows) * per; i += L::workers) {
                            const int s = rows + i / per, ch = i % per, row = step_of(s);
                            asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};" ::"r"(tv + (ch / 8) * kPanel + row * 128 + (((ch & 7) ^ (row & 7)) << 4)), "r"(0) : "memory");
                        }
                    }
                } else {
                    copy_wait<1>();
                }
                if constexpr (!STATE) {
                    tmem_st_wait();
                    if (!TMA || rows < kChunk) tc::fence_proxy_async_smem();
                    tc::fence_before_sync();
                    hand_over<D>(kWeighted);
                }
                // b -> b w as bf16 values.  Where the state leaves, as three, what each leaves rounded to the next: in b's place, in lo, and
                // (once the products with Xb are done) in Xb's place.  Where only Xb is read from it, as two (2^-17): with w = w1 + w2,
                // hi = b w1 rounded, lo = (b w1 - hi) + b w2, where b w1 - hi is exact (16 bits of a product, the first 8 taken away)
                {
                    constexpr int per = D / 8, stride = L::workers / per, turns = kChunk / stride;
                    const int ch = tid % per, row0 = tid / per;
                    const uint32_t off = (ch / 8) * kPanel + row0 * 128 + (((ch & 7) ^ (row0 & 7)) << 4);
                    uint32_t v[turns][4];
                    if (TMA && !STATE) wait(barQK + 8 * slot, phase >> 1);  // (over since A was formed; but it is this wait that shows a thread the copies)
#pragma unroll
                    for (int k = 0; k < turns; ++k)
                        asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v[k][0]), "=r"(v[k][1]), "=r"(v[k][2]), "=r"(v[k][3]) : "r"(tb + off + k * stride * 128) : "memory");
#pragma unroll
                    for (int k = 0; k < turns; ++k) {
                        const uint32_t to = off + k * stride * 128;
                        const int s = step_of(row0 + k * stride);  // its weight in the next state (STATE: in the span's)
                        const bool counts = s < rows && s >= keep_from;
                        const float f = !counts ? 0.f : up_scale * decay_power(g, STATE ? stop - s0 - s : rows - s - less);
                        uint32_t hi[4], lo[4];
                        if (TMA && !counts) v[k][0] = v[k][1] = v[k][2] = v[k][3] = 0u;  // (whatever lies there)
                        if (fine) {
                            const Pair w = twice(f), minus = twice(-1.f);
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                Pair x = mul2(pair_of(v[k][i] << 16, v[k][i] & 0xffff0000u), w);
                                hi[i] = pack2(x.f.x, x.f.y);
                                x = fma2(pair_of(hi[i] << 16, hi[i] & 0xffff0000u), minus, x);
                                lo[i] = pack2(x.f.x, x.f.y);
                                x = fma2(pair_of(lo[i] << 16, lo[i] & 0xffff0000u), minus, x);
                                v[k][i] = pack2(x.f.x, x.f.y);
                                if constexpr (D == 64) v[k][i] = hmul(v[k][i], 0x3f003f00u);  // (it is added twice)
                            }
                        } else {
                            const uint32_t w1 = pack2(f, f);
                            const float rest = f - __uint_as_float(w1 << 16);
                            const uint32_t w2 = pack2(rest, rest);
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                hi[i] = hmul(v[k][i], w1);
                                lo[i] = hfma(v[k][i], w2, hfma(v[k][i], w1, hi[i] ^ 0x80008000u));
                            }
                        }
                        asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(tb + to), "r"(hi[0]), "r"(hi[1]), "r"(hi[2]), "r"(hi[3]) : "memory");
                        asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(base + L::lo + to), "r"(lo[0]), "r"(lo[1]), "r"(lo[2]), "r"(lo[3]) : "memory");
                    }
                    if (fine) {
                        if (!STATE && has_x) wait(barO, phase);
#pragma unroll
                        for (int k = 0; k < turns; ++k)
                            asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(base + L::xb + off + k * stride * 128), "r"(v[k][0]), "r"(v[k][1]), "r"(v[k][2]), "r"(v[k][3]) : "memory");
                    }
                }
                tc::fence_proxy_async_smem();
                tc::fence_before_sync();
                if (!TMA) worker_barrier<D>();  // (their tiles' copies, by all of them)
                hand_over<D>(kReady);
                find_cuts(c + 1);
                if constexpr (!STATE) {
                    // y = O1 + in_scale lambda^step O2, by way of a's tile (32 rows of 64 bytes a warp, 64-byte swizzle) to whole rows
                    const bool sees = !CUT || begin < 0;
                    const uint32_t stage = ta + warp * 2048, own = stage + lane * 64, turn = (lane >> 1) & 3;
                    const Pair w = twice(in_scale * power_of(rate, step));
                    if (!fine || !has_x) wait(barO, phase);
#pragma unroll
                    for (int h = 0; h < (live ? 32 : 0); h += 16) {
                        uint32_t o1[16];
                        __syncwarp();
                        TC_LD16(mine + L::tO1 + col0 + h, o1);
                        if (has_x) {
                            uint32_t o2[16];
                            TC_LD16(mine + L::o2_at(group) + h, o2);
                            tc::tmem_ld_wait();
                            if (sees) {
#pragma unroll
                                for (int i = 0; i < 16; i += 2) {
                                    const Pair v = fma2(pair_of(o2[i], o2[i + 1]), w, pair_of(o1[i], o1[i + 1]));
                                    o1[i] = __float_as_uint(v.f.x), o1[i + 1] = __float_as_uint(v.f.y);
                                }
                            }
                        } else {
                            tc::tmem_ld_wait();
                        }
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            o1[i] = pack2(__uint_as_float(o1[2 * i]), __uint_as_float(o1[2 * i + 1]));
                            if (step < rows) odd = hfma(o1[i], 0u, odd);
                        }
#pragma unroll
                        for (int i = 0; i < 8; i += 4)
                            asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(own + (((h / 8 + i / 4) ^ turn) << 4)), "r"(o1[i]), "r"(o1[i + 1]),
                                         "r"(o1[i + 2]), "r"(o1[i + 3]) : "memory");
                    }
                    if (maps.stores && rows == kChunk) {
                        tc::fence_proxy_async_smem();
                        __syncwarp();
                        if (lane == 0 && col0 < dc) tma_store_4d(&maps.out[m.job], stage, col0, t0 + quad * 32, m.n, m.head);
                    } else if (live) {
                        __syncwarp();
                        const int left = dc - col0 - lane % 4 * 8;
#pragma unroll 1
                        for (int k = 0; k < 4; ++k) {
                            const int r = k * 8 + lane / 4, row = quad * 32 + r;
                            uint32_t v[4];
                            asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
                                         : "r"(stage + r * 64 + (((lane % 4) ^ ((r >> 1) & 3)) << 4)) : "memory");
                            if (step_of(row) < rows && left > 0) {
                                bf16 *const out = py + (long long)(t0 + row) * j.y.t + col0 + lane % 4 * 8;
                                if (j.vec > 1) {
                                    *reinterpret_cast<uint4 *>(out) = make_uint4(v[0], v[1], v[2], v[3]);
                                } else {
#pragma unroll
                                    for (int m = 0; m < 8; ++m)
                                        if (m < left) reinterpret_cast<unsigned short *>(out)[m] = (unsigned short)(v[m / 2] >> (16 * (m & 1)));
                                }
                            }
                        }
                    }
                }
                wait(barX, phase);
                if (*late) in_step(phase);
                if (!TMA) load_c(c + 1);
            }
            bad = (odd & 0x7fff7fffu) != 0;  // (a product with 0 is 0 or NaN)
            if constexpr (!STATE) tma_store_read();
            if constexpr (!TMA) copy_wait<0>();
            // the next item, as the issuing warp noted it (it notes none that is empty), and its state on the way to L2
            taken += chunks > 0;
            Item next{};
            next.at = m.at + (int)gridDim.x;
            if (TMA && notes[(taken & 1) * 16] == next.at) {
                const volatile int *const note = notes + (taken & 1) * 16;
                __threadfence_block();
                next.job = note[1], next.pair = note[2], next.n = note[3], next.head = note[4], next.span = note[5], next.len = note[6];
                next.first = note[7], next.last = note[8], next.stop = note[9], next.chunks = note[10], next.rev = note[11];
                next.g = __int_as_float(note[12]);
            } else {
                next = open(next.at);
            }
            if (!STATE && next.at < items) {
                const decay_job &k = p.job[next.job];
                const float *const s = p.spans > 1 ? k.spans + (long long)next.span * pairs * cells : k.s_in;
                if (s && tid * 32 < cells)  // (a state is as large in every job)
                    asm volatile("prefetch.global.L2 [%0];" ::"l"(s + (long long)next.pair * cells + tid * 32));
            }
            // outputs of padding
            if (!STATE && max(first, stop) < last) {
                const bool wide = j.vec > 1;
                const int per = wide ? dc / 8 : dc, at_once = L::workers / per, r0 = tid / per, c0 = tid - r0 * per;
                if (r0 < at_once)
                    for (int r = max(first, stop) + r0; r < last; r += at_once) {
                        if (wide) *reinterpret_cast<uint4 *>(py + (long long)r * j.y.t + c0 * 8) = make_uint4(0, 0, 0, 0);
                        else py[(long long)r * j.y.t + c0] = __float2bfloat16_rn(0.f);
                    }
            }
            // what leaves: the span's part, or the state itself (of the span that holds the sequence's end)
            float *to = nullptr;
            bool empty = false;
            if constexpr (STATE) {
                to = j.spans + ((long long)m.span * pairs + m.pair) * cells;
                if (tid == 0) p.carry[((long long)m.span * 2 + j.reverse) * pairs + m.pair] = !keeps ? -1.f : decay_power(g, max(0, stop - first));
            } else if (j.s_out) {
                if ((len > first && len <= last) || (len == 0 && m.span == 0)) to = j.s_out + (long long)m.pair * cells;
                empty = j.out_zero && len > 0 && p.reset && p.reset[m.n] != 0;
            }
            if (chunks > 0) {
                if (to) {  // by way of shared memory to whole rows
                    fold(shrink, kept);
#pragma unroll
                    for (int i = 0; i < XN; i += 4) x[state_at<D>(xr, (xc + i) / 4)] = make_float4(X[i], X[i + 1], X[i + 2], X[i + 3]);
                    worker_barrier<D>();
                    bad |= state_out<D>(x, to, da, dc, empty);
                }
                if (bad) {
                    decay_mark(p, m.job, m.pair);
                    if constexpr (STATE)
                        for (int i = 0; i < p.jobs; ++i)  // (another job may read this state)
                            if (p.job[i].spans_t) decay_mark(p, i, m.pair);
                }
            } else if (to) {
                for (int i = tid; i < cells; i += L::workers) {
                    const int r = i / dc, k = i % dc;
                    to[i] = empty || !from ? 0.f : from_t ? from[k * da + r] : from[i];
                }
            }
            done += chunks;
            m = next;
            worker_barrier<D>();  // (tables and places are free)
        }
    }
    tc::fence_before_sync();
    __syncthreads();
    if (!worker && *late) {  // copies and products that were not waited for end before the CTA does
        if (tc::elect_one()) tc::mma_commit(barEnd);
        __syncwarp();
        for (int k = max(0, asked_ab - 2); k < asked_ab; ++k) tc::mbar_wait_bounded(barQK + 8 * (k & 1), (uint32_t)(k >> 1) & 1u, kWait);
        if (asked_c > 0) tc::mbar_wait_bounded(barV, (uint32_t)(asked_c - 1) & 1u, kWait);
        tc::mbar_wait_bounded(barEnd, 0, kWait);
    }
    __syncthreads();
    if (warp == 1) tc::tmem_dealloc(tmem, L::columns);
}

typedef CUresult (*encode_fn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                              const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
encode_fn encoder() {
    static const encode_fn fn = [] {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult q;
        const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q);
        return e == cudaSuccess && q == cudaDriverEntryPointSuccess ? (encode_fn)f : nullptr;
    }();
    return fn;
}

// A map of [T, N, H, dim] whose box is 128 tokens x 64 values of one head (of outputs, 32 x 32); false where a map cannot say it
// (an axis that is broadcast, strides that are not multiples of 16 bytes).
bool make_map(CUtensorMap *m, const decay_array &v, long long T, int N, int H, int dim, bool out) {
    const long long sizes[3] = {T, N, H}, strides[3] = {v.t, v.n, v.h};
    cuuint64_t dims[4] = {(cuuint64_t)dim, (cuuint64_t)T, (cuuint64_t)N, (cuuint64_t)H}, bytes[3];
    for (int i = 0; i < 3; ++i) {
        bytes[i] = sizes[i] == 1 ? 16 : (cuuint64_t)strides[i] * 2;
        if (sizes[i] > 1 && (strides[i] == 0 || strides[i] >= (1ll << 38) || bytes[i] % 16)) return false;
    }
    if ((uintptr_t)v.p % 16 || !encoder()) return false;
    const cuuint32_t box[4] = {out ? 32u : 64u, out ? 32u : (cuuint32_t)kChunk, 1, 1}, one[4] = {1, 1, 1, 1};
    return encoder()(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void *>(v.p), dims, bytes, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                     out ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

int wm_seq_decay_tc_ctas(int Dk, int Dv) { return Dk <= 64 && Dv <= 64 ? 2 : 1; }

void wm_seq_decay_tc_maps(const seq_decay_args &a, const decay_pass &p, decay_maps &maps) {
    const wm_seq_heads *const arrays[4] = {&a.q, &a.k, &a.v, &a.dout};
    maps.use = 1;
    for (int i = 0; i < p.jobs; ++i) maps.use = maps.use && p.job[i].vec > 1;
    for (int i = 0; i < (p.jobs > 1 ? 4 : 3) && maps.use; ++i) {
        const wm_seq_heads &v = *arrays[i];
        maps.use = make_map(&maps.in[i], {v.data, v.stride_t, v.stride_n, v.stride_h}, a.T, a.N, a.H, i < 2 ? a.Dk : a.Dv, false);
    }
    maps.stores = 1;
    for (int i = 0; i < p.jobs && maps.stores; ++i)
        maps.stores = p.job[i].vec > 1 && make_map(&maps.out[i], p.job[i].y, a.T, a.N, a.H, p.job[i].dc, true);
}

namespace {
template <int D, bool STATE, bool TMA, bool CUT>
cudaError_t launch(const decay_pass &p, const decay_maps &maps, unsigned grid, cudaStream_t s) {
    const cudaError_t e = cudaFuncSetAttribute(decay_tc_kernel<D, STATE, TMA, CUT>, cudaFuncAttributeMaxDynamicSharedMemorySize, Plan<D>::bytes);
    if (e != cudaSuccess) return e;
    decay_tc_kernel<D, STATE, TMA, CUT><<<grid, Plan<D>::threads, Plan<D>::bytes, s>>>(p, maps);
    return cudaGetLastError();
}
template <int D, bool STATE>
cudaError_t launch(const decay_pass &p, const decay_maps &maps, unsigned grid, cudaStream_t s) {
    if (maps.use) return p.reset ? launch<D, STATE, true, true>(p, maps, grid, s) : launch<D, STATE, true, false>(p, maps, grid, s);
    return p.reset ? launch<D, STATE, false, true>(p, maps, grid, s) : launch<D, STATE, false, false>(p, maps, grid, s);
}
}  // namespace

cudaError_t wm_seq_decay_tc_launch(wm_seq *h, const decay_pass &p, const decay_maps &maps, bool state, cudaStream_t s) {
    int jobs = 0;
    for (int i = 0; i < p.jobs; ++i) jobs += !(state && p.job[i].spans_t);
    const int D = std::max(p.job[0].da, p.job[0].dc) <= 64 ? 64 : 128;
    const long long items = (long long)p.N * p.H * jobs * p.spans;
    const unsigned grid = (unsigned)std::min(items, (long long)h->sms * (D == 64 ? 2 : 1));
    ++h->last_launches;
    if (D == 64) return state ? launch<64, true>(p, maps, grid, s) : launch<64, false>(p, maps, grid, s);
    return state ? launch<128, true>(p, maps, grid, s) : launch<128, false>(p, maps, grid, s);
}
