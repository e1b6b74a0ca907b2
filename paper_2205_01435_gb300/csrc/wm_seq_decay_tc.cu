// wm_seq_decay_tc.cu -- the decayed linear attention's passes in bf16 on the tensor cores (see wm_seq_decay.cu).
//
// Chunks of 128 tokens, one CTA a job of a head of a sequence (or of a span of it), 256 threads.  For each chunk
//   A = a b^T                     128 x 128, both K-major as they lie in memory
//   P = A * weights               TMEM -> registers -> TMEM as bf16, where the next product reads it
//   O2 = a Xb                     Xb: the state X, fp32 in TMEM, as a bf16 tile
//   O1 = P c,  y = O1 + in_scale lambda^r O2
//   X = lambda^n X + (b w)^T c    in place in TMEM; b w as two bf16 values, so that X is as good as 2^-17 of its terms
// a, b and c lie as [128 tokens][64 values] panels of 128-byte rows in the 128-byte swizzle, which serve as K-major operands
// (a, b in A and O2) and as MN-major ones (c, and b transposed, where the tokens are summed over).  Rows come by asynchronous
// 16-byte copies that a padded token or value leaves as zeros: lengths, strides and either direction of time cost nothing extra.
// Queries and keys are two chunks ahead, values one.
//
// Rounded to bf16: P (each weight of a value by at most 2^-8 of itself, as the output is) and Xb (the state as the queries see
// it); A, O1, O2 and X are fp32.
//
// Masked places hold zeros, and zero times what is not finite is NaN: a chunk whose outputs or state are not finite marks its
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

#define TC_ST32(taddr, r)                                                                                                        \
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "                                                                \
                 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};" \
                 ::"r"((r)[0]), "r"((r)[1]), "r"((r)[2]), "r"((r)[3]), "r"((r)[4]), "r"((r)[5]), "r"((r)[6]), "r"((r)[7]),         \
                   "r"((r)[8]), "r"((r)[9]), "r"((r)[10]), "r"((r)[11]), "r"((r)[12]), "r"((r)[13]), "r"((r)[14]), "r"((r)[15]),   \
                   "r"((r)[16]), "r"((r)[17]), "r"((r)[18]), "r"((r)[19]), "r"((r)[20]), "r"((r)[21]), "r"((r)[22]), "r"((r)[23]), \
                   "r"((r)[24]), "r"((r)[25]), "r"((r)[26]), "r"((r)[27]), "r"((r)[28]), "r"((r)[29]), "r"((r)[30]), "r"((r)[31]), \
                   "r"((uint32_t)(taddr)) : "memory")

namespace {

using bf16 = __nv_bfloat16;

constexpr int kChunk = kDecayTcChunk, kThreads = 256, kPanel = kChunk * 128;  // bytes of 128 tokens x 64 values
constexpr uint32_t kWait = 1u << 22;                                // polls of a wait (each about 20 ns or more)

// What a CTA of head width D (64 or 128) holds: shared memory and TMEM columns.
template <int D>
struct Plan {
    static constexpr int tile = kPanel * (D / 64);
    // (b's tiles and lo are read as operands 128 values wide: with D = 64 the second half is what lies behind them, and unused)
    static constexpr int xb = 0, lo = xb + D * 128 * (D / 64), b = lo + tile, a = b + 2 * tile, c = a + 2 * tile, end = c + tile;
    static constexpr int small = end;  // tables and barriers
    static constexpr int bytes = small + 4 * 132 + 8 * 128 + 48 + 32 + 1024;
    // P lies over A's first columns; with D = 64 O2 over A's others
    static constexpr int tA = 0, tO1 = 128, tO2 = D == 64 ? 64 : 256, tX = D == 64 ? 192 : 384, columns = D == 64 ? 256 : 512;
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
// Two fp32 values at a time.
union Pair {
    unsigned long long u;
    float2 f;
};
__device__ __forceinline__ Pair pair_of(uint32_t a, uint32_t b) {
    Pair p;
    p.f = make_float2(__uint_as_float(a), __uint_as_float(b));
    return p;
}
__device__ __forceinline__ Pair twice(float v) {
    Pair p;
    p.f = make_float2(v, v);
    return p;
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b) {
    Pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.u) : "l"(a.u), "l"(b.u));
    return r;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.u) : "l"(a.u), "l"(b.u), "l"(c.u));
    return r;
}
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

// 128 tokens of an array as swizzled panels.  `at` is the first token's row, step the elements to the next one; rows and values
// that are not there are zeros.  VEC: 16-byte copies.
template <int D, bool VEC>
__device__ __forceinline__ void load_tile(uint32_t dst, const bf16 *at, long long step, int rows, int dim) {
    constexpr int per = D / 8, stride = kThreads / per;
    const int ch = threadIdx.x % per, row0 = threadIdx.x / per, left = dim - ch * 8;
    const bf16 *p = at + row0 * step + ch * 8;
    const uint32_t to = dst + (ch / 8) * kPanel + row0 * 128 + (((ch & 7) ^ (row0 & 7)) << 4);  // (stride is a multiple of 8)
    if (left <= 0) rows = 0;
#pragma unroll
    for (int k = 0; k < kChunk / stride; ++k) {
        const bool on = row0 + k * stride < rows;
        if constexpr (VEC) {
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + k * stride * 128), "l"(on ? p : at), "r"(on ? 16 : 0) : "memory");
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

// VEC: 16-byte accesses; CUT: there may be resets.
template <int D, bool STATE, bool VEC, bool CUT>
__global__ void __launch_bounds__(kThreads, D == 64 ? 2 : 1) decay_tc_kernel(const decay_pass p) {
    using L = Plan<D>;
    extern __shared__ unsigned char raw[];
    unsigned char *smem = raw + ((1024u - (tc::smem_u32(raw) & 1023u)) & 1023u);
    const uint32_t base = tc::smem_u32(smem);
    float *const power = reinterpret_cast<float *>(smem + L::small);        // lambda^0 .. lambda^128
    uint2 *const kept = reinterpret_cast<uint2 *>(power + 132);             // the tokens' weights in the next state: two bf16, each twice
    uint32_t *const cuts = reinterpret_cast<uint32_t *>(kept + 128);        // [2][4]: tokens that begin something new
    int *const late = reinterpret_cast<int *>(cuts + 8);                    // a wait gave up
    uint32_t *const tmem_at = cuts + 9;
    const uint32_t bars = tc::smem_u32(cuts + 12), barA = bars, barO = bars + 8, barX = bars + 16;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, quad = warp & 3, wg = warp >> 2;
    int jobs = 0, at[3] = {};
    for (int i = 0; i < p.jobs; ++i)
        if (!(STATE && p.job[i].spans_t)) at[jobs++] = i;
    const int job = at[blockIdx.x % jobs], span = blockIdx.y;
    const long long pair = blockIdx.x / jobs;
    const decay_job &j = p.job[job];
    const int n = (int)(pair / p.H), head = (int)(pair % p.H), da = j.da, dc = j.dc;
    const decay_seq q = decay_open(p, j, n);
    const float g = p.log_decay[head];
    const long long pairs = (long long)p.N * p.H, cells = (long long)da * dc;
    const long long first = span * p.span_tokens, last = min(p.T, first + p.span_tokens), stop = min(last, q.len);
    const int chunks = stop > first ? (int)((stop - first + kChunk - 1) / kChunk) : 0;

    const bf16 *const pa = static_cast<const bf16 *>(j.a.p) + n * j.a.n + head * j.a.h;
    const bf16 *const pb = static_cast<const bf16 *>(j.b.p) + n * j.b.n + head * j.b.h;
    const bf16 *const pc = static_cast<const bf16 *>(j.c.p) + n * j.c.n + head * j.c.h;
    bf16 *const py = static_cast<bf16 *>(const_cast<void *>(j.y.p)) + n * j.y.n + head * j.y.h;
    const int dir = q.reverse ? -1 : 1;
    const auto load_ab = [&](int c) {  // keys, and queries, of a chunk
        if (c < chunks) {
            const long long s0 = first + (long long)c * kChunk;
            const int rows = (int)min((long long)kChunk, stop - s0), slot = c & 1;
            load_tile<D, VEC>(base + L::b + slot * L::tile, pb + q.at(s0) * j.b.t, dir * j.b.t, rows, da);
            if constexpr (!STATE) load_tile<D, VEC>(base + L::a + slot * L::tile, pa + q.at(s0) * j.a.t, dir * j.a.t, rows, da);
        }
        copy_commit();
    };
    const auto load_c = [&](int c) {
        if (c < chunks) {
            const long long s0 = first + (long long)c * kChunk;
            load_tile<D, VEC>(base + L::c, pc + q.at(s0) * j.c.t, dir * j.c.t, (int)min((long long)kChunk, stop - s0), dc);
        }
        copy_commit();
    };
    const auto find_cuts = [&](int c) {
        if (CUT && warp < 4) {
            const int r = warp * 32 + lane;
            const long long s = first + (long long)c * kChunk + r;
            const unsigned m = __ballot_sync(~0u, c < chunks && s < stop && decay_cut(p, q, s, n));
            if (lane == 0) cuts[(c & 1) * 4 + warp] = m;
        }
    };
    load_ab(0);
    load_c(0);
    load_ab(1);
    find_cuts(0);
    if (tid <= kChunk) power[tid] = decay_power(g, tid);
    if (warp == 0) tc::tmem_alloc(tc::smem_u32(tmem_at), L::columns);
    if (tid == 32) {
        tc::mbar_init(barA, 1);
        tc::mbar_init(barO, 1);
        tc::mbar_init(barX, 1);
        tc::fence_mbar_init();
        *late = 0;
    }
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    const uint32_t tmem = *tmem_at, mine = tmem + ((uint32_t)(quad * 32) << 16);
    const auto wait = [&](uint32_t bar, int c) {
        if (!*(volatile int *)late && !tc::mbar_wait_bounded(bar, (uint32_t)c & 1u, kWait)) {
            *late = 1;
            seq_record(p.status + 1, WM_ERR_TIMEOUT);
        }
        tc::fence_after_sync();
    };

    // the entering state into TMEM: row a thread's lane, half of the columns a warpgroup
    constexpr int W = D / 2;  // columns of X and of the outputs that a thread takes
    const int xrow = quad * 32 + lane, col0 = wg * W;
    const float *from = nullptr;
    int from_t = 0;
    float mul = 1.f;
    if constexpr (!STATE) {
        if (p.spans > 1) {
            from = j.spans + (span * pairs + pair) * cells;
            from_t = j.spans_t;
        } else if (j.s_in) {
            from = j.s_in + pair * cells;
            from_t = j.in_t;
            if (j.first && q.len > 0) mul = power[1];
        }
    }
    bool has_x = from != nullptr && chunks > 0;  // X is not 0
    if (has_x && quad * 32 < D) {
#pragma unroll 1
        for (int h = 0; h < W; h += 32) {
            uint32_t r[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const int col = col0 + h + i;
                float v = 0.f;
                if (xrow < da && col < dc) v = from_t ? from[(long long)col * da + xrow] : from[(long long)xrow * dc + col];
                r[i] = __float_as_uint(mul == 1.f ? v : v * mul);
            }
            __syncwarp();
            TC_ST32(mine + L::tX + col0 + h, r);
        }
        tmem_st_wait();
    }
    uint32_t odd = 0;   // two bf16: NaN once an output was not finite
    bool keeps = true;  // (STATE) no cut so far

#pragma unroll 1
    for (int c = 0; c < chunks; ++c) {
        const long long s0 = first + (long long)c * kChunk;
        const int rows = (int)min((long long)kChunk, stop - s0), slot = c & 1;
        const uint32_t ta = base + L::a + slot * L::tile, tb = base + L::b + slot * L::tile, tv = base + L::c;
        copy_wait<2>();
        tc::fence_proxy_async_smem();
        tc::fence_before_sync();
        __syncthreads();
        if constexpr (!STATE) {
            if (warp == 0 && tc::elect_one()) {
                tc::fence_after_sync();
#pragma unroll
                for (int k = 0; k < D / 16; ++k)
                    tc::mma_bf16(tmem + L::tA, tc::desc_sw128(ta + (k / 4) * kPanel + (k % 4) * 32), tc::desc_sw128(tb + (k / 4) * kPanel + (k % 4) * 32),
                                 tc::idesc_bf16_f32(128, 128), k > 0);
                tc::mma_commit(barA);
            }
            __syncwarp();
        }
        // tokens that begin something new: what a token sees begins with the last of them up to it
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
                    if (cut[i]) keep_from = 32 * i + 31 - __clz(cut[i]);  // (no cuts behind the last row)
                    const uint32_t m = quad > i ? cut[i] : quad < i ? 0u : cut[i] & (~0u >> (31 - lane));
                    if (m) begin = 32 * i + 31 - __clz(m);
                }
            }
        }
        // (time's order, the last token of all: the state leaves as that token wrote it)
        const int less = !STATE && j.first && s0 + rows == q.len ? 1 : 0;
        if (tid < kChunk && (CUT || STATE || c == 0 || rows < kChunk || less)) {
            float w = 0.f;
            if (tid < rows && tid >= keep_from) {
                if constexpr (STATE) w = decay_power(g, stop - s0 - tid);  // up to the span's end
                else w = power[rows - tid - less];
            }
            w *= j.up_scale;
            const float w1 = __bfloat162float(__float2bfloat16_rn(w));
            kept[tid] = make_uint2(pack2(w1, w1), pack2(w - w1, w - w1));
        }
        if constexpr (!STATE) {
            // X -> Xb, and X to what the next state keeps of it
            if (has_x && quad * 32 < D) {
                const Pair shrink = twice(power[rows - less]);
#pragma unroll
                for (int h = 0; h < W; h += 32) {
                    uint32_t r[32];
                    const int col = col0 + h;
                    TC_LD32(mine + L::tX + col, r);
                    tc::tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 32; i += 8) {
                        const float *f = reinterpret_cast<const float *>(r + i);
                        const uint32_t to = base + L::xb + ((col + i) / 64) * (D * 128) + xrow * 128 + (((((col + i) % 64) / 8) ^ (xrow & 7)) << 4);
                        asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(to), "r"(pack2(f[0], f[1])), "r"(pack2(f[2], f[3])),
                                     "r"(pack2(f[4], f[5])), "r"(pack2(f[6], f[7])) : "memory");
                    }
                    if (!CUT || keep_from < 0) {
#pragma unroll
                        for (int i = 0; i < 32; i += 2) {
                            const Pair v = mul2(pair_of(r[i], r[i + 1]), shrink);
                            r[i] = __float_as_uint(v.f.x);
                            r[i + 1] = __float_as_uint(v.f.y);
                        }
                        TC_ST32(mine + L::tX + col, r);
                    }
                }
                tmem_st_wait();
            }
            // A -> P: row xrow, 64 columns a warpgroup, in blocks of 32
            wait(barA, c);
            uint32_t packed[32];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int block = wg * 2 + h, j0 = block * 32;
                if (block > quad) {  // above the diagonal
#pragma unroll
                    for (int i = 0; i < 16; ++i) packed[h * 16 + i] = 0u;
                    continue;
                }
                uint32_t v[32];
                TC_LD32(mine + L::tA + j0, v);
                tc::tmem_ld_wait();
                if (block == quad) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        const float f = __uint_as_float(v[i]) * (j.w_scale * power[max(lane - i, 0)]);
                        v[i] = i <= lane ? __float_as_uint(f) : 0u;
                    }
                } else {  // lambda^(xrow - j0 - 31) lambda^(31 - i): neither is above 1
                    const Pair w = twice(j.w_scale * power[xrow - j0 - 31]);
#pragma unroll
                    for (int i = 0; i < 32; i += 4) {
                        const float4 t = *reinterpret_cast<const float4 *>(power + 28 - i);
                        Pair t0, t1;
                        t0.f = make_float2(t.w, t.z);
                        t1.f = make_float2(t.y, t.x);
                        t0 = mul2(pair_of(v[i], v[i + 1]), mul2(t0, w));
                        t1 = mul2(pair_of(v[i + 2], v[i + 3]), mul2(t1, w));
                        v[i] = __float_as_uint(t0.f.x), v[i + 1] = __float_as_uint(t0.f.y);
                        v[i + 2] = __float_as_uint(t1.f.x), v[i + 3] = __float_as_uint(t1.f.y);
                    }
                }
                if (CUT && any_cut) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] = j0 + i >= begin ? v[i] : 0u;
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) packed[h * 16 + i] = pack2(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1]));
            }
            tc::fence_proxy_async_smem();  // Xb
            tc::fence_before_sync();
            __syncthreads();               // A is read: P and O2 may take its place
            tc::fence_after_sync();
            if (has_x && warp == 0 && tc::elect_one()) {
#pragma unroll
                for (int k = 0; k < D / 16; ++k)
                    tc::mma_bf16(tmem + L::tO2, tc::desc_sw128(ta + (k / 4) * kPanel + (k % 4) * 32), desc_mn(base + L::xb + k * 2048, D * 128),
                                 tc::idesc_bf16_f32(128, D) | kBmn, k > 0);
            }
            __syncwarp();
            TC_ST32(mine + L::tA + wg * 32, packed);
        } else {
            __syncthreads();  // kept
        }
        // b -> b w as two bf16 values, the first in b's place: with w = w1 + w2, hi = b w1 rounded, lo = (b w1 - hi) + b w2,
        // where b w1 - hi is exact (16 bits of a product, the first 8 taken away)
        {
            constexpr int per = D / 8, stride = kThreads / per;
            const int ch = tid % per, row0 = tid / per;
            const uint32_t off = (ch / 8) * kPanel + row0 * 128 + (((ch & 7) ^ (row0 & 7)) << 4);
#pragma unroll
            for (int k = 0; k < kChunk / stride; ++k) {
                const uint32_t to = off + k * stride * 128;
                uint32_t v[4], hi[4], lo[4];
                asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(tb + to));
                const uint2 w = kept[row0 + k * stride];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    hi[i] = hmul(v[i], w.x);
                    lo[i] = hfma(v[i], w.y, hfma(v[i], w.x, hi[i] ^ 0x80008000u));
                }
                asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(tb + to), "r"(hi[0]), "r"(hi[1]), "r"(hi[2]), "r"(hi[3]) : "memory");
                asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(base + L::lo + to), "r"(lo[0]), "r"(lo[1]), "r"(lo[2]), "r"(lo[3]) : "memory");
            }
        }
        if constexpr (!STATE) tmem_st_wait();
        copy_wait<1>();
        tc::fence_proxy_async_smem();
        tc::fence_before_sync();
        __syncthreads();
        const bool onto = STATE ? c > 0 && keep_from < 0 : has_x && keep_from < 0;
        if (warp == 0 && tc::elect_one()) {
            tc::fence_after_sync();
            if constexpr (!STATE) {
#pragma unroll
                for (int k = 0; k < kChunk / 16; ++k)
                    mma_bf16_ts(tmem + L::tO1, tmem + L::tA + k * 8, desc_mn(tv + k * 2048, kPanel), tc::idesc_bf16_f32(128, D) | kBmn, k > 0);
                tc::mma_commit(barO);
            }
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int k = 0; k < kChunk / 16; ++k)
                    tc::mma_bf16(tmem + L::tX, desc_mn((half ? base + L::lo : tb) + k * 2048, kPanel), desc_mn(tv + k * 2048, kPanel),
                                 tc::idesc_bf16_f32(128, D) | kAmn | kBmn, half > 0 || k > 0 || onto);
            tc::mma_commit(barX);
        }
        __syncwarp();
        if constexpr (STATE) keeps = keeps && keep_from < 0;
        find_cuts(c + 1);
        if constexpr (!STATE) {
            // y = O1 + in_scale lambda^r O2
            const Pair w = twice(j.in_scale * power[xrow]);
            const bool sees = !CUT || begin < 0;
            bf16 *const out = py + q.at(s0 + min(xrow, rows - 1)) * j.y.t + col0;
            wait(barO, c);
#pragma unroll
            for (int h = 0; h < W; h += 32) {
                uint32_t o1[32];
                __syncwarp();
                TC_LD32(mine + L::tO1 + col0 + h, o1);
                if (has_x) {
                    uint32_t o2[32];
                    TC_LD32(mine + L::tO2 + col0 + h, o2);
                    tc::tmem_ld_wait();
                    if (sees) {
#pragma unroll
                        for (int i = 0; i < 32; i += 2) {
                            const Pair v = fma2(pair_of(o2[i], o2[i + 1]), w, pair_of(o1[i], o1[i + 1]));
                            o1[i] = __float_as_uint(v.f.x), o1[i + 1] = __float_as_uint(v.f.y);
                        }
                    }
                } else {
                    tc::tmem_ld_wait();
                }
                if (xrow < rows) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        o1[i] = pack2(__uint_as_float(o1[2 * i]), __uint_as_float(o1[2 * i + 1]));
                        odd = hfma(o1[i], 0u, odd);
                    }
                    if constexpr (VEC) {
#pragma unroll
                        for (int i = 0; i < 16; i += 4)
                            if (col0 + h + 2 * i < dc) *reinterpret_cast<uint4 *>(out + h + 2 * i) = make_uint4(o1[i], o1[i + 1], o1[i + 2], o1[i + 3]);
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (col0 + h + i < dc) reinterpret_cast<unsigned short *>(out)[h + i] = (unsigned short)(o1[i / 2] >> (16 * (i & 1)));
                    }
                }
            }
        }
        wait(barX, c);
        has_x = true;
        load_c(c + 1);
        load_ab(c + 2);
    }

    // outputs of padding
    if constexpr (!STATE) {
        const long long pad = max(first, min(q.len, last));
        const int per = VEC ? dc / 8 : dc, at_once = max(1, kThreads / per), r0 = tid / per, c0 = tid - r0 * per;
        if (r0 < at_once)
            for (long long r = pad + r0; r < last; r += at_once) {
                if constexpr (VEC) *reinterpret_cast<uint4 *>(py + r * j.y.t + c0 * 8) = make_uint4(0, 0, 0, 0);
                else py[r * j.y.t + c0] = __float2bfloat16_rn(0.f);
            }
    }
    // what leaves: the span's part, or the state itself (of the span that holds the sequence's end)
    float *to = nullptr;
    bool empty = false;
    if constexpr (STATE) {
        to = j.spans + (span * pairs + pair) * cells;
        if (tid == 0) p.carry[((long long)span * 2 + j.reverse) * pairs + pair] = !keeps ? 0.f : decay_power(g, max(0ll, stop - first));
    } else if (j.s_out) {
        if ((q.len > first && q.len <= last) || (q.len == 0 && span == 0)) to = j.s_out + pair * cells;
        empty = j.out_zero && q.len > 0 && p.reset && p.reset[n] != 0;
    }
    if (chunks > 0) {
        bool bad = (odd & 0x7fff7fffu) != 0;  // (a product with 0 is 0 or NaN)
        if (quad * 32 < D) {
#pragma unroll 1
            for (int h = 0; h < W; h += 32) {
                uint32_t r[32];
                __syncwarp();
                TC_LD32(mine + L::tX + col0 + h, r);
                tc::tmem_ld_wait();
                if (xrow < da) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        const int col = col0 + h + i;
                        const float v = __uint_as_float(r[i]);
                        if (col < dc) {
                            bad |= !(fabsf(v) <= 3.4028235e38f);
                            if (to) to[(long long)xrow * dc + col] = empty ? 0.f : v;
                        }
                    }
                }
            }
        }
        if (bad) {
            decay_mark(p, job, pair);
            if constexpr (STATE)
                for (int i = 0; i < p.jobs; ++i)  // (another job may read this state)
                    if (p.job[i].spans_t) decay_mark(p, i, pair);
        }
    } else if (to) {
        for (long long i = tid; i < cells; i += kThreads) {
            const long long r = i / dc, k = i % dc;
            to[i] = empty || !from ? 0.f : from_t ? from[k * da + r] : from[i];
        }
    }
    copy_wait<0>();
    tc::fence_before_sync();
    __syncthreads();
    if (warp == 0) tc::tmem_dealloc(tmem, L::columns);
}

}  // namespace

int wm_seq_decay_tc_ctas(int Dk, int Dv) { return Dk <= 64 && Dv <= 64 ? 2 : 1; }

namespace {
template <int D, bool STATE, bool VEC, bool CUT>
cudaError_t launch(const decay_pass &p, unsigned grid, cudaStream_t s) {
    const cudaError_t e = cudaFuncSetAttribute(decay_tc_kernel<D, STATE, VEC, CUT>, cudaFuncAttributeMaxDynamicSharedMemorySize, Plan<D>::bytes);
    if (e != cudaSuccess) return e;
    decay_tc_kernel<D, STATE, VEC, CUT><<<dim3(grid, p.spans), kThreads, Plan<D>::bytes, s>>>(p);
    return cudaGetLastError();
}
template <int D, bool STATE>
cudaError_t launch(const decay_pass &p, unsigned grid, cudaStream_t s) {
    bool vec = true;
    for (int i = 0; i < p.jobs; ++i) vec = vec && p.job[i].vec > 1;
    if (vec) return p.reset ? launch<D, STATE, true, true>(p, grid, s) : launch<D, STATE, true, false>(p, grid, s);
    return p.reset ? launch<D, STATE, false, true>(p, grid, s) : launch<D, STATE, false, false>(p, grid, s);
}
}  // namespace

cudaError_t wm_seq_decay_tc_launch(wm_seq *h, const decay_pass &p, bool state, cudaStream_t s) {
    int jobs = 0;
    for (int i = 0; i < p.jobs; ++i) jobs += !(state && p.job[i].spans_t);
    const unsigned grid = (unsigned)((long long)p.N * p.H * jobs);
    ++h->last_launches;
    if (std::max(p.job[0].da, p.job[0].dc) <= 64) return state ? launch<64, true>(p, grid, s) : launch<64, false>(p, grid, s);
    return state ? launch<128, true>(p, grid, s) : launch<128, false>(p, grid, s);
}
