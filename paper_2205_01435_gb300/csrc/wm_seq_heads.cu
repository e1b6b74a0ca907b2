// wm_seq_heads.cu -- the norm of each head's vector and its rotation by position, forward and backward.
//
//   y = x r w, r = 1 / sqrt(mean(x^2) + eps); pairs (a, b) of y turn: (a cos - b sin, b cos + a sin)
//   backward, with d = dy turned back and g = d w: dx = r (g - xhat mean(g xhat)), xhat = x r, dw = sum d xhat
//
// Bound by memory: forward moves 2 values per element, backward 3.  A row (one head of one token) lives in the
// registers of G lanes, each with units of two vectors that hold the two sides of its pairs, so that a rotation
// needs no exchange: halves (vector u and vector u + rotary / (2 VEC)) or neighbours (within a vector).  The angles
// of a tile of tokens are formed once for all heads of the tile, in shared memory.  A CTA works on queries or on keys
// alone: its threads keep their columns' sums of the weight's gradient over all its rows, and a second small launch
// adds the CTAs' sums in a fixed order.
//
// Angles: a frequency is held as a fraction of a turn in 64-bit fixed point (the fp32 value times 1 / 2 pi in fp64),
// and position times that, modulo 2^64, is the angle modulo a turn: its first 32 bits are exact to 2^-32 turns beside the fp64
// rounding of the frequency (position * freq * 2^-53), where position * freq in fp32 is off by whole radians at 10^7.  The functions
// take 24 of them; the other 8 (2^-26 turns) turn the result by the rest (16,384 x 20 x 128: 48.5 -> 49.1 us).
#include <algorithm>

#include "wm_seq_internal.h"

namespace {

constexpr int kThreads = 256;

struct Side {  // queries or keys
    const void *x, *dy;
    void *out;
    long long xt, xn, xh, yt, yn, yh, ot, on, oh;
    const float *w;
    float *part;  // [CTAs][D] sums of the weight's gradient, or NULL
    int heads, ctas;
};

struct HeadArgs {
    Side side[2];
    long long tokens;
    int N, D, rotary;
    int hc, sa, sb;    // units below hc: vectors u sa and u sa + sb turn into one another; the others are two in a row
    int units, group;  // of a row; lanes a row
    int tile;          // tokens that a warp takes at once
    float eps;
    const int32_t *positions;
    const float *freqs;
};

// Rows that a thread has on their way: so many that their loads come to about 32 values.
constexpr int rows_of(int lane_values, bool bwd) { return lane_values <= 4 ? 4 : lane_values <= (bwd ? 8 : 16) ? 2 : 1; }

// The columns' weights of a thread: in registers, or read when they are needed.
template <int VEC, int UPL>
constexpr bool held() {
    return VEC * UPL <= 8;
}

// Vectors of fp32, two values an instruction where there are two.
template <int N>
__device__ __forceinline__ void times(float (&r)[N], const float (&a)[N], const float (&b)[N]) {
    if constexpr (N % 2 == 0) {
#pragma unroll
        for (int m = 0; m < N; m += 2) {
            const seq_pair p = seq_mul2(seq_pair_of(a[m], a[m + 1]), seq_pair_of(b[m], b[m + 1]));
            r[m] = p.f.x, r[m + 1] = p.f.y;
        }
    } else {
#pragma unroll
        for (int m = 0; m < N; ++m) r[m] = a[m] * b[m];
    }
}
template <int N>
__device__ __forceinline__ void times_plus(float (&r)[N], const float (&a)[N], const float (&b)[N], const float (&c)[N]) {  // r = a b + c
    if constexpr (N % 2 == 0) {
#pragma unroll
        for (int m = 0; m < N; m += 2) {
            const seq_pair p = seq_fma2(seq_pair_of(a[m], a[m + 1]), seq_pair_of(b[m], b[m + 1]), seq_pair_of(c[m], c[m + 1]));
            r[m] = p.f.x, r[m + 1] = p.f.y;
        }
    } else {
#pragma unroll
        for (int m = 0; m < N; ++m) r[m] = a[m] * b[m] + c[m];
    }
}
template <int N>
__device__ __forceinline__ void all_of(float (&r)[N], float v) {
#pragma unroll
    for (int m = 0; m < N; ++m) r[m] = v;
}
// Sums of products, in two halves.
template <int N>
__device__ __forceinline__ void dot(seq_pair &sum, const float (&a)[N], const float (&b)[N]) {
    if constexpr (N % 2 == 0) {
#pragma unroll
        for (int m = 0; m < N; m += 2) sum = seq_fma2(seq_pair_of(a[m], a[m + 1]), seq_pair_of(b[m], b[m + 1]), sum);
    } else {
#pragma unroll
        for (int m = 0; m < N; ++m) sum.f.x += a[m] * b[m];
    }
}

// N values that lie side by side, aligned to as many as one access takes.
template <int N>
__device__ __forceinline__ void quads(float (&r)[N], const float *p) {
    constexpr int V = N % 4 == 0 ? 4 : N;
#pragma unroll
    for (int m = 0; m < N; m += V) {
        const seq_vec<float, V> v = seq_load<float, V>(p + m);
#pragma unroll
        for (int k = 0; k < V; ++k) r[m + k] = v.v[k];
    }
}

struct TileRow {  // where a token's rows begin
    long long x, y, o;
};
// Shared memory: phases, two tiles' angles and rows for each warp, weights (and, for their gradient, a row of sums a warp).
constexpr int kWarps = kThreads / 32;
// A token's angles: cosines, sines (as the direction turns), minus those; each a whole number of quads.
__host__ __device__ constexpr int angles(int half) { return 3 * ((half + 3) / 4 * 4); }
struct HeadsSmem {
    size_t turn, row, weight, bytes;
    __host__ __device__ HeadsSmem(int half, int tile, int D, bool backward) {
        turn = ((size_t)half * 8 + 15) / 16 * 16;
        row = (turn + (size_t)kWarps * 2 * tile * angles(half) * 4 + 15) / 16 * 16;
        weight = row + (size_t)kWarps * 2 * tile * sizeof(TileRow);
        bytes = weight + (size_t)(backward ? kWarps : 1) * ((D + 7) / 8 * 8) * 4;
    }
};

// VEC values a vector, UPL units a lane; IN: pairs are neighbours within a vector.
template <class T, int VEC, bool IN, int UPL, bool BWD>
__global__ void __launch_bounds__(kThreads, UPL *VEC > 8 ? 1 : BWD ? 2 : 3) heads_kernel(const __grid_constant__ HeadArgs p) {
    constexpr int R = rows_of(2 * VEC * UPL, BWD);
    constexpr bool HELD = held<VEC, UPL>();
    extern __shared__ __align__(16) unsigned char smem[];
    const int half = p.rotary / 2;
    const HeadsSmem at(half, p.tile, p.D, BWD);
    unsigned long long *phase = reinterpret_cast<unsigned long long *>(smem);
    const int warp = threadIdx.x >> 5, wl = threadIdx.x & 31;
    const int each = angles(half) / 3;
    float *const turns = reinterpret_cast<float *>(smem + at.turn) + (size_t)warp * 2 * p.tile * 3 * each;  // [2][tile][3][each]
    TileRow *const starts = reinterpret_cast<TileRow *>(smem + at.row) + warp * 2 * p.tile;               // [2][tile]
    float *const weight = reinterpret_cast<float *>(smem + at.weight);
    const bool keys = blockIdx.x >= (unsigned)p.side[0].ctas;
    const Side &sd = p.side[keys];
    const int cta = blockIdx.x - (keys ? p.side[0].ctas : 0), heads = sd.heads;
    // the warp's tokens
    const long long w0 = (long long)cta * kWarps + warp, all = (long long)sd.ctas * kWarps;
    long long tok0 = p.tokens * w0 / all;
    const long long end = p.tokens * (w0 + 1) / all;
    for (int i = threadIdx.x; i < half; i += kThreads) {
        const double t = fabs((double)p.freqs[i]) * 0.15915494309189533577;
        const unsigned long long u = __double2ull_rz((t - floor(t)) * 18446744073709551616.0);
        phase[i] = p.freqs[i] < 0.f ? 0ull - u : u;  // (just below a whole turn a small frequency would lose its last bits)
    }
    for (int j = threadIdx.x; j < p.D; j += kThreads) weight[j] = sd.w ? sd.w[j] : 1.f;

    const int lane = wl & (p.group - 1), row0 = wl / p.group, rows_at_once = 32 / p.group;
    const int nv = (p.D + VEC - 1) / VEC;
    int va[UPL], vb[UPL];  // the unit's vectors: their first values
    bool ha[UPL], hb[UPL], turns_here[UPL];
#pragma unroll
    for (int i = 0; i < UPL; ++i) {
        const int u = lane + i * p.group;
        const int a = u < p.hc ? u * p.sa : 2 * p.hc + 2 * (u - p.hc), b = u < p.hc ? a + p.sb : a + 1;
        ha[i] = u < p.units;
        hb[i] = ha[i] && b < nv;
        turns_here[i] = u < p.hc;
        va[i] = ha[i] ? a * VEC : 0;
        vb[i] = hb[i] ? b * VEC : 0;
    }
    // a tile's angles and rows, into the places of even or odd tiles
    // (the positions of the tile after it are on their way meanwhile, a lane each)
    int ahead = half && tok0 + wl < end && wl < p.tile ? p.positions[tok0 + wl] : 0;
    const auto prepare = [&](long long tok0, int slot) {
        const int tile = (int)min((long long)p.tile, end - tok0), now = ahead;
        ahead = half && tok0 + p.tile + wl < end && wl < p.tile ? p.positions[tok0 + p.tile + wl] : 0;
        for (int k = 0; k < tile; ++k) {
            const unsigned long long pos = (unsigned long long)(long long)__shfl_sync(~0u, now, k);
            for (int j = wl; j < half; j += 32) {
                // (the angle's first 24 bits by the functions, what is left of its 32 as a small turn)
                const int angle = (int)((phase[j] * pos + (1ull << 31)) >> 32);
                const float most = (float)angle, rest = (float)(angle - __float2int_rn(most)) * 1.4629180793e-9f;
                float s0, c0;
                sincospif(most * 0x1p-31f, &s0, &c0);
                float sn = fmaf(c0, rest, s0), cs = fmaf(-s0, rest, c0);
                const float f = p.freqs[j];
                if (!(fabsf(f) <= 3.4028235e38f)) sn = cs = f - f;  // NaN: no angle of a frequency that is none
                float *const t = turns + (slot * p.tile + k) * 3 * each + j;
                t[0] = cs;
                t[each] = BWD ? -sn : sn;
                t[2 * each] = BWD ? sn : -sn;
            }
        }
        if (wl < tile) {
            const long long tok = tok0 + wl, t = tok / p.N, n = tok - t * p.N;
            starts[slot * p.tile + wl] = {t * sd.xt + n * sd.xn, t * sd.yt + n * sd.yn, t * sd.ot + n * sd.on};
        }
    };
    __syncthreads();
    if (tok0 < end) prepare(tok0, 0);
    float wa[HELD ? UPL : 1][VEC], wb[HELD ? UPL : 1][VEC];
    const auto weights_of = [&](int i, float(&a)[VEC], float(&b)[VEC]) {
#pragma unroll
        for (int m = 0; m < VEC; ++m) a[m] = weight[va[i] + m], b[m] = weight[vb[i] + m];
    };
    if constexpr (HELD) {
#pragma unroll
        for (int i = 0; i < UPL; ++i) weights_of(i, wa[i], wb[i]);
    }
    float dwa[BWD ? UPL : 1][VEC] = {}, dwb[BWD ? UPL : 1][VEC] = {};
    const float inv_d = 1.f / (float)p.D;
    const int down = rows_at_once / heads, across = rows_at_once - down * heads;  // from a row to the thread's next
    __syncwarp();

    for (int slot = 0; tok0 < end; tok0 += p.tile, slot ^= 1) {
        if (tok0 + p.tile < end) prepare(tok0 + p.tile, slot ^ 1);
        const int tile = (int)min((long long)p.tile, end - tok0), rows = tile * heads;
        const float *const turn = turns + slot * p.tile * 3 * each;
        const TileRow *const start = starts + slot * p.tile;
        int token = row0 / heads, head = row0 - token * heads;
        for (int r = row0; r - row0 < rows; r += R * rows_at_once) {  // (all lanes walk along: they sum over the group)
            seq_vec<T, VEC> xa[R][UPL], xb[R][UPL], ya[BWD ? R : 1][UPL], yb[BWD ? R : 1][UPL];
            T *out[R];
            const float *tw[R];
#pragma unroll
            for (int q = 0; q < R; ++q) {
                const bool on = r + q * rows_at_once < rows;
                const TileRow s = start[on ? token : 0];
                const T *const x = static_cast<const T *>(sd.x) + s.x + (on ? head : 0) * sd.xh;
                const T *const dy = BWD ? static_cast<const T *>(sd.dy) + s.y + (on ? head : 0) * sd.yh : nullptr;
                out[q] = static_cast<T *>(sd.out) + s.o + (on ? head : 0) * sd.oh;
                tw[q] = turn + (on ? token : 0) * 3 * each;
#pragma unroll
                for (int i = 0; i < UPL; ++i) {
                    xa[q][i] = on && ha[i] ? seq_load<T, VEC>(x + va[i]) : seq_vec<T, VEC>{};
                    xb[q][i] = on && hb[i] ? seq_load<T, VEC>(x + vb[i]) : seq_vec<T, VEC>{};
                    if constexpr (BWD) {
                        ya[q][i] = on && ha[i] ? seq_load<T, VEC>(dy + va[i]) : seq_vec<T, VEC>{};
                        yb[q][i] = on && hb[i] ? seq_load<T, VEC>(dy + vb[i]) : seq_vec<T, VEC>{};
                    }
                }
                token += down;
                head += across;
                if (head >= heads) head -= heads, ++token;
            }
#pragma unroll
            for (int q = 0; q < R; ++q) {
                const bool on = r + q * rows_at_once < rows;
                // turns a unit's values in place
                const auto rotate = [&](int i, float(&a)[VEC], float(&b)[VEC]) {
                    if constexpr (IN) {
                        constexpr int C = VEC / 2;
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            float(&v)[VEC] = h ? b : a;
                            const int from = h ? vb[i] : va[i];
                            if (from >= p.rotary) continue;
                            float c[C], s[C];
                            quads(c, tw[q] + from / 2);
                            quads(s, tw[q] + each + from / 2);
#pragma unroll
                            for (int m = 0; m < C; ++m) {
                                const float u = v[2 * m], w = v[2 * m + 1];
                                v[2 * m] = u * c[m] - w * s[m];
                                v[2 * m + 1] = w * c[m] + u * s[m];
                            }
                        }
                    } else if (turns_here[i]) {
                        const float *const t = tw[q] + (lane + i * p.group) * VEC;
                        float c[VEC], s[VEC], n[VEC], p1[VEC], p2[VEC];
                        quads(c, t);
                        quads(s, t + each);
                        quads(n, t + 2 * each);
                        times(p1, b, n);
                        times(p2, a, s);
                        times_plus(a, a, c, p1);
                        times_plus(b, b, c, p2);
                    }
                };
                seq_pair s2 = seq_pair_of(0.f, 0.f), g2 = s2;
                float fa[UPL][VEC], fb[UPL][VEC], da[BWD ? UPL : 1][VEC], db[BWD ? UPL : 1][VEC];
                float ga[BWD ? UPL : 1][VEC], gb[BWD ? UPL : 1][VEC];  // the turned gradient times the weight
#pragma unroll
                for (int i = 0; i < UPL; ++i) {
                    seq_unpack<T, VEC>(xa[q][i], fa[i]);
                    seq_unpack<T, VEC>(xb[q][i], fb[i]);
                    dot(s2, fa[i], fa[i]);
                    dot(s2, fb[i], fb[i]);
                    if constexpr (BWD) {
                        seq_unpack<T, VEC>(ya[q][i], da[i]);
                        seq_unpack<T, VEC>(yb[q][i], db[i]);
                        rotate(i, da[i], db[i]);
                        if constexpr (HELD) {
                            times(ga[i], da[i], wa[i]);
                            times(gb[i], db[i], wb[i]);
                        } else {
                            float ua[VEC], ub[VEC];
                            weights_of(i, ua, ub);
                            times(ga[i], da[i], ua);
                            times(gb[i], db[i], ub);
                        }
                        dot(g2, ga[i], fa[i]);
                        dot(g2, gb[i], fb[i]);
                    }
                }
                float ss = s2.f.x + s2.f.y, gx = g2.f.x + g2.f.y;
                for (int o = p.group / 2; o > 0; o >>= 1) {
                    ss += __shfl_xor_sync(~0u, ss, o);
                    if constexpr (BWD) gx += __shfl_xor_sync(~0u, gx, o);
                }
                const float rs = 1.f / sqrtf(ss * inv_d + p.eps);
                float r[VEC], back[VEC];
                all_of(r, rs);
                all_of(back, BWD ? -rs * (gx * inv_d) : 0.f);
#pragma unroll
                for (int i = 0; i < UPL; ++i) {
                    if constexpr (BWD) {
                        float ta[VEC], tb[VEC];
                        times(ta, fa[i], r);
                        times(tb, fb[i], r);
                        if (on) {  // (of rows that are there: what a thread without one holds may be what it likes)
                            times_plus(dwa[i], da[i], ta, dwa[i]);
                            times_plus(dwb[i], db[i], tb, dwb[i]);
                        }
                        times_plus(fa[i], ta, back, ga[i]);
                        times_plus(fb[i], tb, back, gb[i]);
                        times(fa[i], fa[i], r);
                        times(fb[i], fb[i], r);
                    } else {
                        times(fa[i], fa[i], r);
                        times(fb[i], fb[i], r);
                        if constexpr (HELD) {
                            times(fa[i], fa[i], wa[i]);
                            times(fb[i], fb[i], wb[i]);
                        } else {
                            float ua[VEC], ub[VEC];
                            weights_of(i, ua, ub);
                            times(fa[i], fa[i], ua);
                            times(fb[i], fb[i], ub);
                        }
                        rotate(i, fa[i], fb[i]);
                    }
                    if (on && ha[i]) seq_store<T, VEC>(out[q] + va[i], seq_pack<T, VEC>(fa[i]));
                    if (on && hb[i]) seq_store<T, VEC>(out[q] + vb[i], seq_pack<T, VEC>(fb[i]));
                }
            }
        }
        __syncwarp();  // this tile's places are free, the next one's are there
    }
    if constexpr (BWD) {
        if (!sd.part) return;
        // over a warp's row groups by halves, then the warps one after the other (in the weights' place)
        __syncthreads();
        float *const sums = weight + warp * ((p.D + 7) / 8 * 8);
#pragma unroll
        for (int i = 0; i < UPL; ++i)
#pragma unroll
            for (int m = 0; m < VEC; ++m) {
                for (int o = 16; o >= p.group; o >>= 1) {
                    dwa[i][m] += __shfl_xor_sync(~0u, dwa[i][m], o);
                    dwb[i][m] += __shfl_xor_sync(~0u, dwb[i][m], o);
                }
                if (wl < p.group) {
                    if (ha[i]) sums[va[i] + m] = dwa[i][m];
                    if (hb[i]) sums[vb[i] + m] = dwb[i][m];
                }
            }
        __syncthreads();
        for (int j = threadIdx.x; j < p.D; j += kThreads) {
            float v = weight[j];
            for (int w = 1; w < kThreads / 32; ++w) v += weight[w * ((p.D + 7) / 8 * 8) + j];
            sd.part[(long long)cta * p.D + j] = v;
        }
    }
}

// dweight[j] = sum of the CTAs' parts: 8 columns a block, 32 stretches of CTAs.
__global__ void __launch_bounds__(256) heads_weight_kernel(const float *part0, const float *part1, int ctas0, int ctas1, int D,
                                                           float *dw0, float *dw1) {
    __shared__ float sum[32][8];
    const bool keys = blockIdx.y;
    const float *part = keys ? part1 : part0;
    float *dw = keys ? dw1 : dw0;
    const int ctas = keys ? ctas1 : ctas0, x = threadIdx.x & 7, y = threadIdx.x >> 3, j = blockIdx.x * 8 + x;
    if (!dw) return;
    float v = 0.f;
    if (j < D) {
#pragma unroll 4
        for (int c = y; c < ctas; c += 32) v += part[(long long)c * D + j];
    }
    sum[y][x] = v;
    __syncthreads();
    if (y == 0 && j < D) {
        for (int k = 1; k < 32; ++k) v += sum[k][x];
        dw[j] = v;
    }
}

bool aligned(const wm_seq_heads &v, const seq_heads_args &a, int heads, size_t bytes, size_t es) {
    return (uintptr_t)v.data % bytes == 0 && (a.T == 1 || v.stride_t * es % bytes == 0) && (a.N == 1 || v.stride_n * es % bytes == 0) &&
           (heads == 1 || v.stride_h * es % bytes == 0);
}

// Values an access moves: as many as 16 bytes hold, where rows and the pairs' halves are whole vectors.
int vector_of(const seq_heads_args &a, bool backward) {
    const int es = a.dtype == WM_BF16 ? 2 : 4;
    for (int vec = 16 / es; vec > 1; vec >>= 1) {
        bool ok = a.D % vec == 0 && (a.interleaved ? a.rotary : a.rotary / 2) % vec == 0;
        for (int i = 0; i < 2 && ok; ++i)
            if (a.heads[i] > 0)
                ok = aligned(a.x[i], a, a.heads[i], vec * es, es) && aligned(a.out[i], a, a.heads[i], vec * es, es) &&
                     (!backward || aligned(a.dy[i], a, a.heads[i], vec * es, es));
        if (ok) return vec;
    }
    return 1;
}

// CTAs of queries and keys: as many as run at once, shared by their heads, no more than their warps have tokens.
void ctas_of(const wm_seq *h, const seq_heads_args &a, bool backward, int (&ctas)[2]) {
    const int all = a.heads[0] + a.heads[1], room = (backward ? 2 : 3) * h->sms;
    const long long tokens = a.T * a.N;
    for (int i = 0; i < 2; ++i) {
        const long long share = a.heads[i] ? std::max(1ll, (long long)room * a.heads[i] / all) : 0;
        ctas[i] = (int)std::min(share, std::max(a.heads[i] ? 1ll : 0, (tokens + kWarps - 1) / kWarps));
    }
}

// Tokens a warp takes at once: about 16 rows a lane group.
int tile_of(const seq_heads_args &a, int group) {
    const int heads = std::max(a.heads[0], a.heads[1]), want = std::max(1, 16 * (32 / group) / heads);
    const int room = a.rotary ? std::max(1, 1024 / a.rotary) : 32;  // 100 KB of angles
    return std::min({want, room, 32});
}

template <class T, int VEC, bool IN, int UPL>
cudaError_t run(wm_seq *h, const HeadArgs &p, bool backward, cudaStream_t s) {
    const size_t bytes = HeadsSmem(p.rotary / 2, p.tile, p.D, backward).bytes;
    cudaError_t e = cudaSuccess;
    if (bytes > 48 << 10)
        e = backward ? cudaFuncSetAttribute(heads_kernel<T, VEC, IN, UPL, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes)
                     : cudaFuncSetAttribute(heads_kernel<T, VEC, IN, UPL, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e != cudaSuccess) return e;
    const unsigned grid = (unsigned)(p.side[0].ctas + p.side[1].ctas);
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = s;
    ++h->last_launches;
    return backward ? cudaLaunchKernelEx(&cfg, heads_kernel<T, VEC, IN, UPL, true>, p)
                    : cudaLaunchKernelEx(&cfg, heads_kernel<T, VEC, IN, UPL, false>, p);
}

template <class T, int VEC, bool IN>
cudaError_t run_units(wm_seq *h, HeadArgs &p, const seq_heads_args &a, bool backward, cudaStream_t s) {
    // (a lane holds up to 8 values of each of a unit's vectors, 4 where it loads them one by one)
    constexpr int most = VEC >= 8 ? 1 : VEC == 4 ? 2 : 4;
    int g = 1;
    while (g < 32 && p.units > most * g) g <<= 1;
    p.group = g;
    p.tile = tile_of(a, g);
    const int upl = (p.units + g - 1) / g;
    if (upl <= 1) return run<T, VEC, IN, 1>(h, p, backward, s);
    if constexpr (VEC <= 4 || sizeof(T) == 2) {
        if (upl <= 2) return run<T, VEC, IN, 2>(h, p, backward, s);
    }
    if constexpr (VEC <= 2) {
        if (upl <= 3) return run<T, VEC, IN, 3>(h, p, backward, s);
    }
    if constexpr (VEC <= 4) {
        if (upl <= 4) return run<T, VEC, IN, 4>(h, p, backward, s);
    }
    if constexpr (VEC <= 2) {
        if (upl <= 8) return run<T, VEC, IN, 8>(h, p, backward, s);
    }
    if constexpr (VEC == 1) {
        if (upl <= 16) return run<T, VEC, IN, 16>(h, p, backward, s);
    }
    return cudaErrorInvalidValue;  // (D <= 1024 needs none)
}

template <class T>
cudaError_t run_type(wm_seq *h, HeadArgs &p, const seq_heads_args &a, bool backward, cudaStream_t s) {
    const int vec = vector_of(a, backward), nv = (a.D + vec - 1) / vec;
    const bool in = a.interleaved && vec > 1;
    p.hc = in ? 0 : a.rotary / 2 / vec;
    p.sa = a.interleaved ? 2 : 1;
    p.sb = a.interleaved ? 1 : p.hc;
    p.units = p.hc + (nv - 2 * p.hc + 1) / 2;
    if constexpr (sizeof(T) == 2) {
        if (vec == 8) return in ? run_units<T, 8, true>(h, p, a, backward, s) : run_units<T, 8, false>(h, p, a, backward, s);
    }
    if (vec == 4) return in ? run_units<T, 4, true>(h, p, a, backward, s) : run_units<T, 4, false>(h, p, a, backward, s);
    if (vec == 2) return in ? run_units<T, 2, true>(h, p, a, backward, s) : run_units<T, 2, false>(h, p, a, backward, s);
    return run_units<T, 1, false>(h, p, a, backward, s);
}

}  // namespace

size_t wm_seq_heads_backward_ws(const wm_seq *h, const seq_heads_args &a) {
    if (!a.dweight[0] && !a.dweight[1]) return 0;
    int ctas[2];
    ctas_of(h, a, true, ctas);
    return (size_t)(ctas[0] + ctas[1]) * a.D * 4;
}

cudaError_t wm_seq_heads_launch(wm_seq *h, const seq_heads_args &a, bool backward, cudaStream_t s) {
    h->last_launches = 0;
    HeadArgs p{};
    p.tokens = a.T * a.N;
    p.N = a.N; p.D = a.D; p.rotary = a.rotary; p.eps = a.eps;
    p.positions = a.positions; p.freqs = a.freqs;
    int ctas[2];
    ctas_of(h, a, backward, ctas);
    for (int i = 0; i < 2; ++i) {
        Side &d = p.side[i];
        d.heads = a.heads[i];
        d.ctas = ctas[i];
        d.x = a.x[i].data; d.xt = a.x[i].stride_t; d.xn = a.x[i].stride_n; d.xh = a.x[i].stride_h;
        d.dy = a.dy[i].data; d.yt = a.dy[i].stride_t; d.yn = a.dy[i].stride_n; d.yh = a.dy[i].stride_h;
        d.out = a.out[i].data; d.ot = a.out[i].stride_t; d.on = a.out[i].stride_n; d.oh = a.out[i].stride_h;
        d.w = a.weight[i];
        d.part = backward && a.dweight[i] ? static_cast<float *>(h->ws) + (i ? (size_t)ctas[0] * a.D : 0) : nullptr;
    }
    cudaError_t e = cudaSuccess;
    if (p.tokens > 0) e = a.dtype == WM_BF16 ? run_type<__nv_bfloat16>(h, p, a, backward, s) : run_type<float>(h, p, a, backward, s);
    if (e != cudaSuccess || !backward || (!a.dweight[0] && !a.dweight[1])) return e;
    if (p.tokens == 0) ctas[0] = ctas[1] = 0;  // (no rows: sums of nothing)
    ++h->last_launches;
    heads_weight_kernel<<<dim3((a.D + 7) / 8, 2), 256, 0, s>>>(p.side[0].part, p.side[1].part, ctas[0], ctas[1], a.D, a.dweight[0],
                                                                 a.dweight[1]);
    return cudaGetLastError();
}
