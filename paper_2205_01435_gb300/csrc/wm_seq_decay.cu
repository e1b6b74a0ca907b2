// wm_seq_decay.cu -- linear attention whose weights decay with the distance: fp32 kernels, single tokens, launches.
//
//   S_t = lambda S_{t-1} + k_t v_t^T,  o_t = scale S_t^T q_t
//
// Chunks of C tokens: within a chunk the products of queries and keys are formed, weighted by lambda^(i-j) and multiplied
// by the values; what came before the chunk enters through the state X alone.  That is 2 C (Dk + Dv) operations a token
// within the chunk and 4 Dk Dv with the state, where the recurrence takes 5 Dk Dv on a state that would have to be moved
// for every token.
//
// The gradients are three passes of the same form.  With X the state, dq_t = scale X_t dout_t is the attention of queries
// dout, keys v and values k (its state is X transposed).  Against the order of time, G_t = scale q_t dout_t^T +
// lambda G_{t+1} is a state with keys q and values dout: dv_t = G_t^T k_t reads it with queries k, and dk_t = G_t v_t reads
// its transpose with queries v.  One launch runs the three side by side, a sequence's three passes next to one another, so
// that two of the three reads of an array come from L2.
//
// Few sequences: each is cut into spans of time that run side by side.  A first launch forms what each span's own tokens
// give the state (no queries, no outputs), a second joins them along time, the third is the pass itself.
#include <algorithm>

#include "wm_seq_decay.cuh"

namespace {

constexpr int kChunk = 64, kSlice = 64, kThreads = 256;

__device__ __forceinline__ float4 ld4(const float *p) { return *reinterpret_cast<const float4 *>(p); }

// ------------------------------------------------------------------ chunks in fp32
// A CTA: one sequence of one head, one job, kSlice values of c.  Every product sums over the quads of two tiles' rows, so that a
// thread's 4 x 4 outputs take 8 quads from shared memory and 32 instructions of two multiply-adds for 64 of them: c and the
// weighted b are turned over on the way, the state is held as [values of c][values of a].  (128 x 128 x 8 x 64, forward: 205 us
// with one multiply-add an instruction and rows read across.)
// What bounds it (128 x 128 x 8 x 64: 135 us forward, 362 backward; 100 x 200 x 7 x 43 ragged 109 and 281): reads of shared memory
// (57% of its cycles), instructions (50%) and multiply-adds (39%) together, at the 16 warps that two CTAs of 100 KB hold.  More warps
// with smaller blocks read more: 512 threads of 4 x 2 outputs 152 and 422 us.  Taking both products with a's rows at once saves
// reads, but not registers: 141 and 372.
// A tile: rows of ld floats (a multiple of 32), the quads of row r turned by r & 7: 8 rows' quads of one column lie in 8 places.
__device__ __forceinline__ int quad_at(int r, int quad, int ld) { return r * ld + ((quad ^ (r & 7)) << 2); }
__device__ __forceinline__ int cell_at(int r, int c, int ld) { return quad_at(r, c >> 2, ld) + (c & 3); }

template <int LD>  // values of a row of a, b and x: 64, 128 or 256
struct ChunkTiles {
    static constexpr bool apart = LD < 256;  // the weighted b has a place of its own, and the next chunk comes while the state is formed
    float *a, *b, *bt, *c, *p, *x, *kept, *power;
    __device__ explicit ChunkTiles(float *m) {
        a = m;                                // [64][LD]
        b = a + kChunk * LD;                  // [64][LD]
        c = b + kChunk * LD;                  // turned over: [64 values][64 tokens]
        p = c + kSlice * kChunk;              // [64][64]: c as it comes, then the products
        x = p + kChunk * kChunk;              // [64 values of c][LD]
        kept = x + kSlice * LD;
        power = kept + kChunk;                // lambda^0 .. lambda^64
        bt = apart ? power + kChunk + 4 : a;  // the weighted b turned over, [LD][64]; or, once a is read, in its place
    }
    static constexpr size_t bytes =
        sizeof(float) * (2 * kChunk * LD + kSlice * kChunk + kChunk * kChunk + kSlice * LD + kChunk + kChunk + 4 + (apart ? kChunk * LD : 0));
};

// Rows [0, rows) of a chunk, D values from column col0, zeros around: on their way in fp32 (copy_commit, copy_wait), there in bf16.
template <class T, int ld>
__device__ __forceinline__ void load_rows(float *dst, const decay_array &g, long long base, const decay_seq &q, long long s0, int rows, int col0, int D,
                                          int vec) {
    const T *const first = static_cast<const T *>(g.p) + base + q.at(s0) * g.t + col0;
    const long long next = q.reverse ? -g.t : g.t;
    constexpr bool fp32 = sizeof(T) == 4;
    if (vec > 1) {  // 16 bytes
        constexpr int V = 16 / sizeof(T), per = ld / V, turns = kChunk * per / kThreads, at_once = kThreads / per;
        const int d = threadIdx.x % per * V, r0 = threadIdx.x / per;
#pragma unroll 4
        for (int i = 0; i < turns; ++i) {
            const int r = r0 + i * at_once;
            const bool on = r < rows && d < D;
            const T *const at = first + (on ? r * next + d : 0);
            if constexpr (fp32) {
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst + quad_at(r, d / 4, ld))), "l"(at),
                             "r"(on ? 16 : 0) : "memory");
            } else {
                float f[V] = {};
                if (on) seq_unpack<T, V>(seq_load<T, V>(at), f);
#pragma unroll
                for (int k = 0; k < V; k += 4) *reinterpret_cast<float4 *>(dst + quad_at(r, (d + k) / 4, ld)) = make_float4(f[k], f[k + 1], f[k + 2], f[k + 3]);
            }
        }
    } else {
        for (int r = threadIdx.x >> 5; r < kChunk; r += kThreads / 32) {
#pragma unroll
            for (int d = threadIdx.x & 31; d < ld; d += 32) {
                const bool on = r < rows && d < D;
                const T *const at = first + (on ? r * next + d : 0);
                if constexpr (fp32)
                    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst + cell_at(r, d, ld))), "l"(at),
                                 "r"(on ? 4 : 0) : "memory");
                else
                    dst[cell_at(r, d, ld)] = on ? seq_to_float(*at) : 0.f;
            }
        }
    }
}

// acc[i][k] += sums over `quads` quads of rows r0 + i of u and rows c0 + 16 k of v, for k < B.  (r0 a multiple of 4.  The quads of
// rows 16 apart are turned alike: one address for all k, the rest in the instructions; quads are taken 4 at a time, those behind
// the last are zeros.)
template <int LDU, int LDV, int B>
__device__ __forceinline__ void products(seq_pair (&acc)[4][4], const float *u, int r0, const float *v, int c0, int quads) {
    const char *const ub = reinterpret_cast<const char *>(u + r0 * LDU), *const vb = reinterpret_cast<const char *>(v + c0 * LDV);
    const int ut = (r0 & 7) << 4, vt = (c0 & 7) << 4;
#pragma unroll 1
    for (int d0 = 0; d0 < quads << 4; d0 += 64) {
#pragma unroll
        for (int e = 0; e < 64; e += 16) {
            float4 x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const float4 *>(ub + ((d0 | e) ^ ut ^ (i << 4)) + i * LDU * 4);
            const char *const y0 = vb + ((d0 | e) ^ vt);
#pragma unroll
            for (int k = 0; k < B; ++k) {
                const float4 y = *reinterpret_cast<const float4 *>(y0 + k * 16 * LDV * 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    acc[i][k] = seq_fma2(seq_pair_of(x[i].x, x[i].y), seq_pair_of(y.x, y.y), acc[i][k]);
                    acc[i][k] = seq_fma2(seq_pair_of(x[i].z, x[i].w), seq_pair_of(y.z, y.w), acc[i][k]);
                }
            }
        }
    }
}
template <int LDU, int LDV>
__device__ __forceinline__ void products(seq_pair (&acc)[4][4], const float *u, int r0, const float *v, int c0, int quads, int blocks) {
    if (blocks == 4) products<LDU, LDV, 4>(acc, u, r0, v, c0, quads);
    else if (blocks == 3) products<LDU, LDV, 3>(acc, u, r0, v, c0, quads);
    else if (blocks == 2) products<LDU, LDV, 2>(acc, u, r0, v, c0, quads);
    else products<LDU, LDV, 1>(acc, u, r0, v, c0, quads);
}

// STATE: only what the span's tokens give the state.
template <class T, bool STATE, int LD>
__device__ __forceinline__ void decay_chunks(const decay_pass &p, int item, float *smem, unsigned (&cuts)[2]) {
    int job = 0, slice = item;
    long long pair = 0;
    {
        int per = 0, before[3];
        for (int i = 0; i < p.jobs; ++i) {
            before[i] = per;
            per += STATE && p.job[i].spans_t ? 0 : (p.job[i].dc + kSlice - 1) / kSlice;
        }
        pair = slice / per;
        slice -= (int)pair * per;
        for (int i = 1; i < p.jobs; ++i)
            if (slice >= before[i] && !(STATE && p.job[i].spans_t)) job = i;
        slice -= before[job];
    }
    const decay_job &j = p.job[job];
    if (p.only_redo && !p.redo[1 + job * (long long)p.N * p.H + pair]) return;
    __syncthreads();  // (an item before this one is done with the shared memory)
    const int n = (int)(pair / p.H), head = (int)(pair % p.H), span = blockIdx.y, da = j.da, dq = (da + 3) / 4;
    const int col0 = slice * kSlice, cols = min(kSlice, j.dc - col0);
    const ChunkTiles<LD> m(smem);
    const decay_seq q = decay_open(p, j, n);
    const float g = p.log_decay[head];
    // Rows 4 ty and on, columns tx and on by 16.  Later rows see more tokens: a quarter of the processor, which has warps w and w + 4,
    // takes 8 rows of the first half and the 8 as far from the end (128 x 128 x 8 x 64: forward 141 -> 135 us, backward 381 -> 362).
    const int tid = threadIdx.x, wy = tid & 128 ? 11 - (tid >> 5) : tid >> 5, tx = tid & 15, ty = wy * 2 + (tid >> 4 & 1);
    const long long pairs = (long long)p.N * p.H, cells = (long long)da * j.dc;
    const long long first = span * p.span_tokens, last = min(p.T, first + p.span_tokens);
    const int cblocks = (cols + 15) / 16;  // of 16 values of c

    // the entering state
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
            if (j.first && q.len > 0) mul = decay_power(g, 1);
        }
    }
    if (!from) {
        for (int i = tid; i < LD * kSlice / 4; i += kThreads) reinterpret_cast<float4 *>(m.x)[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    } else {
#pragma unroll 8
        for (int i = tid; i < LD * kSlice; i += kThreads) {
            // (value of a, of c: lanes along what lies side by side)
            const int r = from_t ? i % LD : i / kSlice, c = from_t ? i / LD : i % kSlice;
            float v = 0.f;
            if (r < da && c < cols) v = (from_t ? from[(long long)(col0 + c) * da + r] : from[(long long)r * j.dc + col0 + c]);
            m.x[cell_at(c, r, LD)] = mul == 1.f ? v : v * mul;
        }
    }
    if (tid <= kChunk) m.power[tid] = decay_power(g, tid);
    float carry = 1.f;

    const long long an = n * j.a.n + head * j.a.h, bn = n * j.b.n + head * j.b.h, cn = n * j.c.n + head * j.c.h;
    const auto rows_of = [&](long long s0) { return (int)max(0ll, min((long long)kChunk, min(last, q.len) - s0)); };
    const auto load = [&](long long s0) {
        const int rows = rows_of(s0);
        if (rows > 0) {
            load_rows<T, LD>(m.b, j.b, bn, q, s0, rows, 0, da, j.vec);
            load_rows<T, kSlice>(m.p, j.c, cn, q, s0, rows, col0, cols, j.vec);
            if constexpr (!STATE) load_rows<T, LD>(m.a, j.a, an, q, s0, rows, 0, da, j.vec);
        }
        copy_commit();
    };
    load(first);
    const float w_scale = j.w_scale, in_scale = j.in_scale, up_scale = j.up_scale;
    T *const y0 = static_cast<T *>(const_cast<void *>(j.y.p)) + n * j.y.n + head * j.y.h + col0;
    for (long long s0 = first; s0 < last; s0 += kChunk) {
        const int rows = rows_of(s0);
        if (rows == 0) {
            if constexpr (STATE) break;
            const int pad = (int)min((long long)kChunk, last - s0);
            for (int r = tid >> 5; r < pad; r += kThreads / 32)
                for (int c = tid & 31; c < cols; c += 32) y0[(s0 + r) * j.y.t + c] = seq_from_float<T>(0.f);
            continue;
        }
        if (tid < 64) {
            const unsigned c = __ballot_sync(~0u, decay_cut(p, q, s0 + tid, n, g) && tid < rows);
            if ((tid & 31) == 0) cuts[tid >> 5] = c;
        }
        copy_wait<0>();
        __syncthreads();  // 1: the tiles are there
        const unsigned long long cut = cuts[0] | (unsigned long long)cuts[1] << 32;
        // the first token that token i sees; with none of the chunk cut before, the state too
        auto start = [&](int i) {
            const unsigned long long c = cut & (~0ull >> (63 - i));
            return c ? 63 - __clzll((long long)c) : -1;
        };
        const int keep_from = start(rows - 1);
        // (time's order, the last chunk of all: the state leaves as the last token wrote it)
        const int less = j.first && s0 + rows == q.len && !STATE ? 1 : 0;
        if (tid < kChunk) m.kept[tid] = tid < rows && tid >= keep_from ? up_scale * m.power[rows - tid - less] : 0.f;
        // rows [64][ld] -> [ld][64], each row times its weight (rows that are not there or cut off: zeros, whatever they hold; a weight
        // that has become 0 keeps what is not finite); true if a value is not finite
        const auto turn = [&](float *to, const float *rowsm, int ld, const float *w) {
            float odd = 0.f;
            const int r = tid % kChunk;
            const float f = w ? w[r] : 1.f;
            const bool none = w && !(r < rows && r >= keep_from);
#pragma unroll 4
            for (int d = tid / kChunk; d < ld / 4; d += kThreads / kChunk) {
                float4 v = ld4(rowsm + quad_at(r, d, ld));
                odd += v.x * 0.f + v.y * 0.f + v.z * 0.f + v.w * 0.f;
                if (w) v = none ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(v.x * f, v.y * f, v.z * f, v.w * f);
                to[cell_at(4 * d, r, kChunk)] = v.x;
                to[cell_at(4 * d + 1, r, kChunk)] = v.y;
                to[cell_at(4 * d + 2, r, kChunk)] = v.z;
                to[cell_at(4 * d + 3, r, kChunk)] = v.w;
            }
            return !(odd == 0.f);
        };
        bool careful = turn(m.c, m.p, kSlice, nullptr);  // (zero weights would make NaN of what is not finite)

        if constexpr (!STATE) {
            int begin[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) begin[i] = start(ty * 4 + i);
            // p = a b^T, weighted; columns beyond the rows' own are not seen
            seq_pair acc[4][4] = {};
            const bool live = ty * 4 < rows;  // (of four rows, any)
            if (live) products<LD, LD>(acc, m.a, ty * 4, m.b, tx, dq, ty / 4 + 1);
            careful = __syncthreads_or(careful);  // 2: c is turned over, and p's place free
            if constexpr (m.apart) careful |= turn(m.bt, m.b, LD, m.kept);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = ty * 4 + i;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int c = tx + 16 * k;
                    const bool seen = c <= r && c >= begin[i] && r < rows;
                    m.p[cell_at(r, c, kChunk)] = seen ? (acc[i][k].f.x + acc[i][k].f.y) * (w_scale * m.power[r - c]) : 0.f;
                }
            }
            careful = __syncthreads_or(careful);  // 3
            // y = lambda^r X^T a + p c
            float y[4][4];
            {
                seq_pair in[4][4] = {};
                if (live) products<LD, LD>(in, m.a, ty * 4, m.x, tx, dq, cblocks);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float w = in_scale * m.power[ty * 4 + i];
#pragma unroll
                    for (int h = 0; h < 4; ++h) y[i][h] = begin[i] < 0 ? w * (in[i][h].f.x + in[i][h].f.y) : 0.f;
                }
            }
            if (!careful) {
                seq_pair own[4][4] = {};
                if (live) products<kChunk, kChunk>(own, m.p, ty * 4, m.c, tx, ty + 1, cblocks);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int h = 0; h < 4; ++h) y[i][h] += own[i][h].f.x + own[i][h].f.y;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    for (int k = max(begin[i], 0); k <= min(ty * 4 + i, rows - 1); ++k) {
                        const float w = m.p[cell_at(ty * 4 + i, k, kChunk)];
#pragma unroll
                        for (int h = 0; h < 4; ++h) y[i][h] += w * m.c[cell_at(tx + 16 * h, k, kChunk)];
                    }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = ty * 4 + i;
                if (s0 + r >= last) continue;
                T *const out = y0 + q.at(s0 + r) * j.y.t + tx;
#pragma unroll
                for (int h = 0; h < 4; ++h)
                    if (tx + 16 * h < cols) out[16 * h] = seq_from_float<T>(r >= rows ? 0.f : y[i][h]);
            }
        }
        if constexpr (STATE || !m.apart) {
            __syncthreads();  // (kept is there, a and p are read)
            const bool odd = turn(m.bt, m.b, LD, m.kept) || careful;
            careful = __syncthreads_or(odd);
        } else {
            __syncthreads();  // 4: the state is read
        }
        if constexpr (m.apart) load(s0 + kChunk);
        // X = lambda^n X + (kept b)^T c
        const float shrink = m.power[rows - less];
        if (ty * 4 < cols)
            for (int r0 = 0; r0 < da; r0 += 64) {
                seq_pair acc[4][4] = {};
                const int blocks = min(4, (da - r0 + 15) / 16);
                if (!careful) {
                    products<kChunk, kChunk>(acc, m.c, ty * 4, m.bt + r0 * kChunk, tx, (rows + 3) / 4, blocks);
                } else {
                    for (int k = max(keep_from, 0); k < rows; ++k) {
                        float v[4];
#pragma unroll
                        for (int h = 0; h < 4; ++h) v[h] = h < blocks ? m.bt[cell_at(r0 + tx + 16 * h, k, kChunk)] : 0.f;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float u = m.c[cell_at(ty * 4 + i, k, kChunk)];
#pragma unroll
                            for (int h = 0; h < 4; ++h) acc[i][h].f.x += u * v[h];
                        }
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
                        const int r = r0 + tx + 16 * h;
                        if (r >= LD) break;
                        float *const x = m.x + cell_at(ty * 4 + i, r, LD);
                        const float v = acc[i][h].f.x + acc[i][h].f.y;
                        *x = keep_from < 0 ? *x * shrink + v : v;
                    }
            }
        carry = keep_from >= 0 || carry < 0.f ? -1.f : carry * shrink;
        if constexpr (!m.apart) {
            __syncthreads();
            load(s0 + kChunk);
        }
    }
    copy_wait<0>();
    __syncthreads();
    // what leaves: the span's part, or the state itself (of the span that holds the sequence's end)
    float *to = nullptr;
    bool empty = false;
    if constexpr (STATE) {
        to = j.spans + (span * pairs + pair) * cells;
        if (slice == 0 && tid == 0) p.carry[((long long)span * 2 + j.reverse) * pairs + pair] = carry;
    } else if (j.s_out) {
        const bool ends = q.len > first && q.len <= last;
        if (ends || (q.len == 0 && span == 0)) to = j.s_out + pair * cells;
        empty = j.out_zero && q.len > 0 && ((p.reset && p.reset[n] != 0) || decay_keeps_none(g));
    }
    if (to)
#pragma unroll 8
        for (int i = tid; i < LD * kSlice; i += kThreads) {
            const int r = i / kSlice, c = i % kSlice;
            if (r < da && c < cols) to[(long long)r * j.dc + col0 + c] = empty ? 0.f : m.x[cell_at(c, r, LD)];
        }
}

template <class T, bool STATE, int LD>
__global__ void __launch_bounds__(kThreads, LD == 64 ? 2 : 1) decay_chunk_kernel(const __grid_constant__ decay_pass p, int items) {
    extern __shared__ __align__(16) float smem[];
    __shared__ unsigned cuts[2];  // the chunk's tokens that begin something new
    if (p.only_redo && *p.redo == 0) return;
    for (long long i = blockIdx.x; i < items; i += gridDim.x) decay_chunks<T, STATE, LD>(p, (int)i, smem, cuts);
}

// Spans' own parts -> what enters each span, along time.  A thread takes one cell of a state (QUAD: four), the parts of 8
// spans on their way at a time; jobs that form the spans.
template <int QUAD>
__global__ void __launch_bounds__(256) decay_join_kernel(const decay_pass p) {
    const decay_job &j = p.job[blockIdx.y];
    if (j.spans_t) return;
    const long long cells = (long long)j.da * j.dc, pairs = (long long)p.N * p.H, i = ((long long)blockIdx.x * 256 + threadIdx.x) * QUAD;
    if (i >= cells * pairs) return;
    const long long pair = i / cells, cell = i % cells;
    float x[QUAD] = {};
    if (j.s_in) {
        const int n = (int)(pair / p.H);
        const float mul = j.first && (!p.lengths || p.lengths[n] > 0) ? decay_power(p.log_decay[pair % p.H], 1) : 1.f;
#pragma unroll
        for (int k = 0; k < QUAD; ++k) {
            const long long r = (cell + k) / j.dc, c = (cell + k) % j.dc;
            x[k] = j.s_in[pair * cells + (j.in_t ? c * j.da + r : cell + k)];
            if (mul != 1.f) x[k] *= mul;
        }
    }
    using V = seq_vec<float, QUAD>;
    const float *const carry = p.carry + (long long)j.reverse * pairs + pair;
    for (int s = 0; s < p.spans; s += 8) {
        V own[8];
        float c[8];
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (s + k < p.spans) {
                own[k] = seq_load<float, QUAD>(j.spans + (s + k) * pairs * cells + i);
                c[k] = carry[(s + k) * 2 * pairs];
            }
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (s + k < p.spans) {
                V v;
#pragma unroll
                for (int h = 0; h < QUAD; ++h) {
                    v.v[h] = x[h];
                    x[h] = c[k] < 0.f ? own[k].v[h] : x[h] * c[k] + own[k].v[h];
                }
                seq_store<float, QUAD>(j.spans + (s + k) * pairs * cells + i, v);
            }
    }
}

// ------------------------------------------------------------------ token by token
// Up to a few tokens: the state in registers, read and written once.  A CTA: one head of one sequence, 4 CT columns of its
// state; thread (row group, column group) holds rows of 4 columns.
struct StepArgs {
    decay_array q, k, v, o;
    int T, N, H, Dk, Dv, ct, slices, vec;
    const float *log_decay, *s0;
    const uint8_t *reset;
    const int32_t *lengths;
    float scale, *s_last;
    int *status;
};

template <class T, int ROWS, bool VEC>
__global__ void __launch_bounds__(256, ROWS <= 4 ? 6 : ROWS <= 8 ? 4 : 2) decay_step_kernel(const __grid_constant__ StepArgs p) {
    __shared__ float4 quads[16];  // of the values, which are read four at a time
    __shared__ float q[256], k[256];
    float *const v = reinterpret_cast<float *>(quads);
    __shared__ float part[8][64];
    const int item = (int)blockIdx.x, at_pair = p.slices == 1 ? item : item / p.slices, slice = item - at_pair * p.slices;  // (below 2^30)
    const int n = at_pair / p.H, head = at_pair - n * p.H, tid = threadIdx.x;
    const long long pair = at_pair;
    const int shift = p.ct == 16 ? 4 : 3, cg = tid & (p.ct - 1), rg = tid >> shift, groups = 256 >> shift, width = 4 << shift, col0 = slice * width,
              col = col0 + cg * 4;
    int len = p.T;
    if (p.lengths) {
        len = p.lengths[n];
        if (len < 0 || len > p.T) seq_record(p.status, WM_ERR_INVALID_ARG);
        len = max(0, min(len, p.T));
    }
    float x[ROWS][4];
    // (a first token that a reset begins does not see the state)
    const bool read = p.s0 && !(len > 0 && p.reset && p.reset[n]);
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int r = rg + i * groups;
#pragma unroll
        for (int h = 0; h < 4; ++h) x[i][h] = 0.f;
        if (!read || r >= p.Dk) continue;
        const float *at = p.s0 + (pair * p.Dk + r) * p.Dv + col;
        if constexpr (VEC) {
            if (col < p.Dv) {
                const float4 u = ld4(at);
                x[i][0] = u.x, x[i][1] = u.y, x[i][2] = u.z, x[i][3] = u.w;
            }
        } else {
#pragma unroll
            for (int h = 0; h < 4; ++h)
                if (col + h < p.Dv) x[i][h] = at[h];
        }
    }
    const float keep = expf(p.log_decay[head]);
    const bool alone = decay_keeps_none(p.log_decay[head]);
    for (int t = 0; t < p.T; ++t) {
        T *out = static_cast<T *>(const_cast<void *>(p.o.p)) + t * p.o.t + n * p.o.n + head * p.o.h;
        if (t >= len) {
            if (tid < width && col0 + tid < p.Dv) out[col0 + tid] = seq_from_float<T>(0.f);
            continue;
        }
        if (tid < p.Dk) {
            q[tid] = seq_to_float(static_cast<const T *>(p.q.p)[t * p.q.t + n * p.q.n + head * p.q.h + tid]);
            k[tid] = seq_to_float(static_cast<const T *>(p.k.p)[t * p.k.t + n * p.k.n + head * p.k.h + tid]);
        }
        if (tid < width)
            v[tid] = col0 + tid < p.Dv ? seq_to_float(static_cast<const T *>(p.v.p)[t * p.v.t + n * p.v.n + head * p.v.h + col0 + tid]) : 0.f;
        const bool cut = alone || (p.reset && p.reset[(long long)t * p.N + n]);
        __syncthreads();
        const float4 w = quads[cg];
        float y[4] = {};
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const int r = rg + i * groups;
            if (r >= p.Dk) break;
            const float a = k[r], b = q[r];
            x[i][0] = (cut ? 0.f : keep * x[i][0]) + a * w.x;
            x[i][1] = (cut ? 0.f : keep * x[i][1]) + a * w.y;
            x[i][2] = (cut ? 0.f : keep * x[i][2]) + a * w.z;
            x[i][3] = (cut ? 0.f : keep * x[i][3]) + a * w.w;
#pragma unroll
            for (int h = 0; h < 4; ++h) y[h] += b * x[i][h];
        }
        for (int o = 16; o >= p.ct; o >>= 1)
#pragma unroll
            for (int h = 0; h < 4; ++h) y[h] += __shfl_xor_sync(~0u, y[h], o);
        if ((tid & 31) < p.ct)
#pragma unroll
            for (int h = 0; h < 4; ++h) part[tid >> 5][cg * 4 + h] = y[h];
        __syncthreads();
        if (tid < width && col0 + tid < p.Dv) {
            float sum = part[0][tid];
#pragma unroll
            for (int g = 1; g < 8; ++g) sum += part[g][tid];
            out[col0 + tid] = seq_from_float<T>(sum * p.scale);
        }
    }
    if (!p.s_last) return;
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int r = rg + i * groups;
        if (r >= p.Dk) break;
        float *at = p.s_last + (pair * p.Dk + r) * p.Dv + col;
        if constexpr (VEC) {
            if (col < p.Dv) *reinterpret_cast<float4 *>(at) = make_float4(x[i][0], x[i][1], x[i][2], x[i][3]);
        } else {
#pragma unroll
            for (int h = 0; h < 4; ++h)
                if (col + h < p.Dv) at[h] = x[i][h];
        }
    }
}

// ------------------------------------------------------------------ launches
decay_array array_of(const wm_seq_heads &v) { return {v.data, v.stride_t, v.stride_n, v.stride_h}; }

bool aligned16(const decay_array &v, const seq_decay_args &a, int D) {
    const long long es = a.dtype == WM_BF16 ? 2 : 4;
    return (uintptr_t)v.p % 16 == 0 && D * es % 16 == 0 && (a.T == 1 || v.t * es % 16 == 0) && (a.N == 1 || v.n * es % 16 == 0) &&
           (a.H == 1 || v.h * es % 16 == 0);
}

// The jobs of a call: the pass itself, or the gradients' three.
decay_pass pass_of(const wm_seq *h, const seq_decay_args &a, bool backward) {
    decay_pass p{};
    p.T = a.T; p.N = a.N; p.H = a.H;
    p.log_decay = a.log_decay; p.reset = a.reset; p.lengths = a.lengths;
    p.status = h->status;
    const decay_array q = array_of(a.q), k = array_of(a.k), v = array_of(a.v), o = array_of(a.o), dout = array_of(a.dout);
    const decay_array in[4] = {q, k, v, dout};
    const auto job = [&](int ia, int ib, int ic, const decay_array &out, int da, int dc) {
        decay_job j{};
        const decay_array &x = in[ia], &y = in[ib], &z = in[ic];
        j.a = x; j.b = y; j.c = z; j.y = out;
        j.map[0] = ia; j.map[1] = ib; j.map[2] = ic;
        j.da = da; j.dc = dc;
        j.w_scale = j.in_scale = a.scale;
        j.up_scale = 1.f;
        const int V = a.dtype == WM_BF16 ? 8 : 4;
        j.vec = aligned16(x, a, da) && aligned16(y, a, da) && aligned16(z, a, dc) && aligned16(out, a, dc) ? V : 1;
        return j;
    };
    if (!backward) {
        p.jobs = 1;
        decay_job &f = p.job[0] = job(0, 1, 2, o, a.Dk, a.Dv);
        f.first = f.fine = 1;
        f.s_in = a.s0;
        f.s_out = a.s_last;
        return p;
    }
    p.jobs = 3;
    decay_job &dq = p.job[0] = job(3, 2, 1, array_of(a.dq), a.Dv, a.Dk);
    dq.first = 1;
    dq.s_in = a.s0;
    dq.in_t = 1;
    decay_job &dv = p.job[1] = job(1, 0, 3, array_of(a.dv), a.Dk, a.Dv);
    dv.reverse = dv.fine = 1;
    dv.in_scale = 1.f;
    dv.up_scale = a.scale;
    dv.s_in = a.ds_last;
    dv.s_out = a.ds0;
    dv.out_zero = 1;
    decay_job &dk = p.job[2] = job(2, 3, 0, array_of(a.dk), a.Dv, a.Dk);
    dk.reverse = 1;
    dk.in_scale = 1.f;
    dk.up_scale = a.scale;
    dk.s_in = a.ds_last;
    dk.in_t = 1;
    dk.spans_t = 1;
    return p;
}

int slices_of(int dc) { return (dc + kSlice - 1) / kSlice; }

// Few sequences are cut into spans of time, of at least 4 chunks, as many as take the least time by this count.  A launch takes
// (chunks of a span + what opening and leaving one takes) for each round of CTAs that the SMs hold, in fp32 0.6 of it for a last
// round of one CTA an SM where two fit; with spans the launch that forms their states comes on top, at 0.57 of a pass (0.4 in fp32).
// Measured, us, spans in brackets, the chosen one first (no resets, heads that lose 1/8 to 1/1024 a token).  bf16: 65,536 x 1 x 8 x 128 x 64,
// forward 213 (19), 587 (6), 232 (38), backward 487 (19), 589 (6), 507 (38); 8192 x 2 x 8 x 128, forward 92 (9), 100 (16), 137 (4);
// 8192 x 4 x 16 x 64, forward 143 (4), 222 (1), 147 (8), backward 284 (1), 309 (3); 16,384 x 1 x 16 x 64, backward 163 (19), 176 (6), 178 (12).
// fp32: 4096 x 24 x 8 x 64, forward 981 (3), 1068 (1), 1020 (8), backward 2092 (1), 2571 (3); 8192 x 1 x 4 x 128, forward 195 (19), 233 (32),
// backward 485 (19), 542 (12).
void split(const wm_seq *h, decay_pass &p, const seq_decay_args &a, bool tc) {
    long long ctas = 0, state_ctas = 0;
    int da = 0;
    for (int i = 0; i < p.jobs; ++i) {
        const int n = tc ? 1 : slices_of(p.job[i].dc);
        ctas += n;
        if (!p.job[i].spans_t) state_ctas += n;
        da = std::max(da, p.job[i].da);
    }
    ctas *= (long long)p.N * p.H;
    state_ctas *= (long long)p.N * p.H;
    const int chunk = tc ? kDecayTcChunk : kChunk, held = tc ? wm_seq_decay_tc_ctas(a.Dk, a.Dv) : da <= 64 ? 2 : 1, room = h->sms * held;
    const double opening = tc ? 2.0 : 0.5, of_a_pass = tc ? 0.57 : 0.4;
    const auto rounds = [&](long long n) {
        const long long rest = n % room;
        return (double)(n / room) + (rest == 0 ? 0.0 : !tc && held == 2 && rest <= h->sms ? 0.6 : 1.0);
    };
    const long long chunks = (p.T + chunk - 1) / chunk, most = std::min({chunks / 4, 4 * room / std::max(1ll, ctas) + 1, 65535ll});
    long long spans = 1, per = std::max(1ll, chunks);
    double least = rounds(ctas) * (double)(chunks + opening);
    for (long long s = 2; s <= most; ++s) {
        const long long chunks_of = (chunks + s - 1) / s, n = (chunks + chunks_of - 1) / chunks_of;
        const double time = (rounds(ctas * n) + of_a_pass * rounds(state_ctas * n)) * ((double)chunks_of + opening);
        if (time < least) least = time, spans = n, per = chunks_of;
    }
    p.span_tokens = per * chunk;
    p.spans = (int)spans;
}

// Tensor cores: bf16, heads of up to 128 values.
bool tc_takes(const seq_decay_args &a) { return a.dtype == WM_BF16 && a.Dk <= kDecayTcMost && a.Dv <= kDecayTcMost; }

// Up to how many tokens go one by one (both ways measured, us, state in place).  bf16 on tensor cores: 256 heads x 64 x 64, 12 tokens:
// steps 25, chunks 25; 16: 31 and 25; 16,384 heads, 12: 422 and 466; 16: 548 and 461.  fp32, 4096 heads, 32: 292 and 316; 256 heads,
// 12: 27 and 29; 16: 31 and 29.
bool steps_take(const wm_seq *h, const seq_decay_args &a, bool backward) {
    return !backward && a.T <= (tc_takes(a) ? 12 : (long long)a.N * a.H >= 2ll * h->sms ? 32 : 14);
}

// Scratch of a pass: the spans' states and carries, the marks of what is taken again, a copy of an entering state whose place
// the leaving one takes.
struct Scratch {
    size_t spans[3] = {}, carry = 0, copy = 0, redo = 0, bytes = 0;
    // (the gradients: two jobs read ds_last, one writes ds0; tensor cores: a sequence may be taken again from s0)
    static bool copies(const seq_decay_args &a, bool backward, bool tc) {
        return backward ? a.ds0 && a.ds0 == a.ds_last : tc && a.s_last && a.s_last == a.s0;
    }
    Scratch(const decay_pass &p, const seq_decay_args &a, bool backward, bool tc) {
        const auto take = [&](size_t n) {
            const size_t at = bytes;
            bytes += (n + 255) / 256 * 256;
            return at;
        };
        const size_t pairs = (size_t)p.N * p.H;
        if (p.spans > 1) {
            for (int i = 0; i < p.jobs; ++i)
                if (!p.job[i].spans_t) spans[i] = take(pairs * p.spans * p.job[i].da * p.job[i].dc * 4);
            carry = take(pairs * p.spans * 2 * 4);
        }
        if (copies(a, backward, tc)) copy = take(pairs * a.Dk * a.Dv * 4);
        if (tc) redo = take((1 + p.jobs * pairs) * 4);
    }
};

template <class T, int ROWS>
cudaError_t run_steps(wm_seq *h, const StepArgs &p, cudaStream_t s) {
    const unsigned grid = (unsigned)((long long)p.N * p.H * p.slices);
    ++h->last_launches;
    if (p.vec) decay_step_kernel<T, ROWS, true><<<grid, 256, 0, s>>>(p);
    else decay_step_kernel<T, ROWS, false><<<grid, 256, 0, s>>>(p);
    return cudaGetLastError();
}

template <class T>
cudaError_t steps(wm_seq *h, const seq_decay_args &a, cudaStream_t s) {
    StepArgs p{};
    p.q = array_of(a.q); p.k = array_of(a.k); p.v = array_of(a.v); p.o = array_of(a.o);
    p.T = (int)a.T; p.N = a.N; p.H = a.H; p.Dk = a.Dk; p.Dv = a.Dv;
    p.log_decay = a.log_decay; p.s0 = a.s0; p.reset = a.reset; p.lengths = a.lengths;
    p.scale = a.scale; p.s_last = a.s_last; p.status = h->status;
    // 64 columns a CTA, 32 where that leaves SMs without one
    const long long pairs = (long long)a.N * a.H;
    p.ct = a.Dv <= 32 || pairs * ((a.Dv + 63) / 64) < h->sms ? 8 : 16;
    p.slices = (a.Dv + 4 * p.ct - 1) / (4 * p.ct);
    p.vec = a.Dv % 4 == 0 && (uintptr_t)a.s0 % 16 == 0 && (uintptr_t)a.s_last % 16 == 0;
    const int groups = 256 / p.ct, rows = (a.Dk + groups - 1) / groups;
    if (rows <= 2) return run_steps<T, 2>(h, p, s);
    if (rows <= 4) return run_steps<T, 4>(h, p, s);
    if (rows <= 8) return run_steps<T, 8>(h, p, s);
    return run_steps<T, 16>(h, p, s);
}

int items_of(const decay_pass &p, bool state) {
    int n = 0;
    for (int i = 0; i < p.jobs; ++i) n += state && p.job[i].spans_t ? 0 : slices_of(p.job[i].dc);
    return (int)((long long)p.N * p.H * n);
}

template <class T, bool STATE, int LD>
cudaError_t chunk_launch(wm_seq *h, const decay_pass &p, cudaStream_t s) {
    constexpr int bytes = (int)ChunkTiles<LD>::bytes;
    const cudaError_t e = cudaFuncSetAttribute(decay_chunk_kernel<T, STATE, LD>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != cudaSuccess) return e;
    const int items = items_of(p, STATE);
    ++h->last_launches;
    decay_chunk_kernel<T, STATE, LD><<<dim3((unsigned)(p.only_redo ? std::min(items, h->sms) : items), p.spans), kThreads, bytes, s>>>(p, items);
    return cudaGetLastError();
}
template <class T, bool STATE>
cudaError_t chunk_launch(wm_seq *h, const decay_pass &p, cudaStream_t s) {
    int da = 0;
    for (int i = 0; i < p.jobs; ++i) da = std::max(da, p.job[i].da);
    if (da <= 64) return chunk_launch<T, STATE, 64>(h, p, s);
    return da <= 128 ? chunk_launch<T, STATE, 128>(h, p, s) : chunk_launch<T, STATE, 256>(h, p, s);
}

// The pass, on tensor cores or in fp32; in spans, what each gives the state and the joins first.
template <class T>
cudaError_t run_pass(wm_seq *h, const seq_decay_args &a, decay_pass &p, bool tc, cudaStream_t s) {
    const long long pairs = (long long)p.N * p.H;
    cudaError_t e;
    decay_maps maps;
    if (tc) {
        wm_seq_decay_tc_maps(a, p, maps);
        p.test_wait = h->test_wait;  // (an injected wait goes to the call's first such launch)
        h->test_wait = 0;
    }
    if (tc && (e = cudaMemsetAsync(p.redo, 0, (size_t)(1 + p.jobs * pairs) * 4, s)) != cudaSuccess) return e;
    if (p.spans > 1) {
        e = tc ? wm_seq_decay_tc_launch(h, p, maps, true, s) : chunk_launch<T, true>(h, p, s);
        if (e != cudaSuccess) return e;
        p.test_wait = 0;
        const long long cells = pairs * a.Dk * a.Dv;
        ++h->last_launches;
        if ((long long)a.Dk * a.Dv % 4 == 0) decay_join_kernel<4><<<dim3((unsigned)((cells / 4 + 255) / 256), p.jobs), 256, 0, s>>>(p);
        else decay_join_kernel<1><<<dim3((unsigned)((cells + 255) / 256), p.jobs), 256, 0, s>>>(p);
        if ((e = cudaGetLastError()) != cudaSuccess) return e;
    }
    if (!tc) return chunk_launch<T, false>(h, p, s);
    if ((e = wm_seq_decay_tc_launch(h, p, maps, false, s)) != cudaSuccess) return e;
    p.only_redo = 1;
    p.spans = 1;
    p.span_tokens = (p.T + kChunk - 1) / kChunk * kChunk;
    return chunk_launch<T, false>(h, p, s);
}


}  // namespace

size_t wm_seq_decay_ws(const wm_seq *h, const seq_decay_args &a, bool backward) {
    if (a.T == 0 || steps_take(h, a, backward)) return 0;
    decay_pass p = pass_of(h, a, backward);
    split(h, p, a, tc_takes(a));
    return Scratch(p, a, backward, tc_takes(a)).bytes;
}

cudaError_t wm_seq_decay_launch(wm_seq *h, const seq_decay_args &a, bool backward, cudaStream_t s) {
    h->last_launches = 0;
    const size_t state = (size_t)a.N * a.H * a.Dk * a.Dv * 4;
    if (a.T == 0) {  // the state, or its gradient, goes through
        float *to = backward ? a.ds0 : a.s_last;
        const float *from = backward ? a.ds_last : a.s0;
        if (!to || to == from) return cudaSuccess;
        return from ? cudaMemcpyAsync(to, from, state, cudaMemcpyDeviceToDevice, s) : cudaMemsetAsync(to, 0, state, s);
    }
    if (steps_take(h, a, backward)) return a.dtype == WM_BF16 ? steps<__nv_bfloat16>(h, a, s) : steps<float>(h, a, s);
    const bool tc = tc_takes(a);
    decay_pass p = pass_of(h, a, backward);
    split(h, p, a, tc);
    const Scratch w(p, a, backward, tc);
    unsigned char *ws = static_cast<unsigned char *>(h->ws);
    for (int i = 0; i < p.jobs; ++i)
        if (p.spans > 1) p.job[i].spans = reinterpret_cast<float *>(ws + w.spans[p.job[i].spans_t ? 1 : i]);
    p.carry = reinterpret_cast<float *>(ws + w.carry);
    p.redo = reinterpret_cast<int *>(ws + w.redo);
    if (Scratch::copies(a, backward, tc)) {
        float *copy = reinterpret_cast<float *>(ws + w.copy);
        const cudaError_t e = cudaMemcpyAsync(copy, backward ? a.ds_last : a.s0, state, cudaMemcpyDeviceToDevice, s);
        if (e != cudaSuccess) return e;
        (backward ? p.job[1].s_in : p.job[0].s_in) = copy;
        if (backward) p.job[2].s_in = copy;
    }
    return a.dtype == WM_BF16 ? run_pass<__nv_bfloat16>(h, a, p, tc, s) : run_pass<float>(h, a, p, tc, s);
}
