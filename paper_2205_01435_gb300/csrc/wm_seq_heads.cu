// wm_seq_heads.cu -- the norm of each head's vector and its rotation by position, forward and backward.
//
//   y = x r w, r = 1 / sqrt(mean(x^2) + eps); pairs (a, b) of y turn: (a cos - b sin, b cos + a sin)
//   backward, with d = dy turned back and g = d w: dx = r (g - x r^2 mean(g x)), dw = sum d x r
//
// Bound by memory: forward moves 2 values per element, backward 3.  A row (one head of one token) lives in the
// registers of G lanes, each with units of two vectors that hold the two sides of its pairs, so that a rotation
// needs no exchange: halves (vector u and vector u + rotary / (2 VEC)) or neighbours (within a vector).  The angles
// of a tile of tokens are formed once for all heads of the tile, in shared memory.  A CTA works on queries or on keys
// alone: its threads keep their columns' sums of the weight's gradient over all its rows, and a second small launch
// adds the CTAs' sums in a fixed order.
//
// Angles: a frequency is held as a fraction of a turn in 64-bit fixed point (the fp32 value times 1 / 2 pi in fp64),
// and position times that, modulo 2^64, is the angle modulo a turn: exact to 2^-33 turns beside the fp64 rounding of
// the frequency (position * freq * 2^-53), where position * freq in fp32 is off by whole radians at 10^7.
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
    int tile;          // tokens
    float eps;
    const int32_t *positions;
    const float *freqs;
};

// How a row is cut: vectors of VEC values; IN: pairs are neighbours within a vector.
template <class T, int VEC, bool IN, int UPL, bool BWD>
__global__ void __launch_bounds__(kThreads, UPL *VEC >= 16 ? 1 : BWD ? 2 : 4) heads_kernel(const HeadArgs p) {
    extern __shared__ __align__(16) unsigned char smem[];
    const int half = p.rotary / 2;
    unsigned long long *phase = reinterpret_cast<unsigned long long *>(smem);
    float2 *turn = reinterpret_cast<float2 *>(phase + half);                    // [tile][half]: cos, sin
    float *weight = reinterpret_cast<float *>(turn + (size_t)p.tile * half);    // [D], padded to whole vectors
    const bool keys = blockIdx.x >= (unsigned)p.side[0].ctas;
    const Side &sd = p.side[keys];
    const int cta = blockIdx.x - (keys ? p.side[0].ctas : 0);
    for (int i = threadIdx.x; i < half; i += kThreads) {
        const double turns = (double)p.freqs[i] * 0.15915494309189533577;
        phase[i] = __double2ull_rz((turns - floor(turns)) * 18446744073709551616.0);
    }
    for (int j = threadIdx.x; j < p.D; j += kThreads) weight[j] = sd.w ? sd.w[j] : 1.f;

    const int lane = threadIdx.x & (p.group - 1), row0 = threadIdx.x / p.group, rows_at_once = kThreads / p.group;
    const int nv = (p.D + VEC - 1) / VEC;
    int va[UPL], vb[UPL];  // the unit's vectors; -1: none
#pragma unroll
    for (int i = 0; i < UPL; ++i) {
        const int u = lane + i * p.group;
        va[i] = vb[i] = -1;
        if (u < p.units) {
            va[i] = u < p.hc ? u * p.sa : 2 * p.hc + 2 * (u - p.hc);
            vb[i] = u < p.hc ? va[i] + p.sb : va[i] + 1;
            if (vb[i] >= nv) vb[i] = -1;
        }
    }
    float dwa[BWD ? UPL : 1][VEC] = {}, dwb[BWD ? UPL : 1][VEC] = {};
    const float inv_d = 1.f / (float)p.D;
    const bool sums = BWD && sd.part;

    for (long long tok0 = (long long)cta * p.tile; tok0 < p.tokens; tok0 += (long long)sd.ctas * p.tile) {
        const int tile = (int)min((long long)p.tile, p.tokens - tok0);
        __syncthreads();  // the angles of the tile before are read; weights and phases are there
        for (int i = threadIdx.x; i < tile * half; i += kThreads) {
            const int k = i / half, j = i - k * half;
            const unsigned long long ph = phase[j] * (unsigned long long)(long long)p.positions[tok0 + k];
            float sn, cs;
            sincospif((float)(int)((ph + (1ull << 31)) >> 32) * 0x1p-31f, &sn, &cs);
            const float f = p.freqs[j];
            if (!(fabsf(f) <= 3.4028235e38f)) sn = cs = f - f;  // NaN: no angle of a frequency that is none
            turn[i] = make_float2(cs, sn);
        }
        __syncthreads();
        const int rows = tile * sd.heads;
        for (int r0 = 0; r0 < rows; r0 += rows_at_once) {  // (all lanes walk along: they sum over the group)
            const int r = r0 + row0;
            const bool on = r < rows;
            const int k = on ? r / sd.heads : 0, head = on ? r - k * sd.heads : 0;
            const long long tok = tok0 + k, t = tok / p.N, n = tok - t * p.N;
            const T *x = static_cast<const T *>(sd.x) + t * sd.xt + n * sd.xn + head * sd.xh;
            const T *dy = BWD ? static_cast<const T *>(sd.dy) + t * sd.yt + n * sd.yn + head * sd.yh : nullptr;
            T *out = static_cast<T *>(sd.out) + t * sd.ot + n * sd.on + head * sd.oh;
            const float2 *tw = turn + k * half;
            seq_vec<T, VEC> xa[UPL], xb[UPL], ya[BWD ? UPL : 1], yb[BWD ? UPL : 1];
#pragma unroll
            for (int i = 0; i < UPL; ++i) {
                const bool a = on && va[i] >= 0, b = on && vb[i] >= 0;
                xa[i] = a ? seq_load<T, VEC>(x + va[i] * VEC) : seq_vec<T, VEC>{};
                xb[i] = b ? seq_load<T, VEC>(x + vb[i] * VEC) : seq_vec<T, VEC>{};
                if constexpr (BWD) {
                    ya[i] = a ? seq_load<T, VEC>(dy + va[i] * VEC) : seq_vec<T, VEC>{};
                    yb[i] = b ? seq_load<T, VEC>(dy + vb[i] * VEC) : seq_vec<T, VEC>{};
                }
            }
            // turns a unit's values in place, by sign * angle
            auto rotate = [&](int i, float(&a)[VEC], float(&b)[VEC], float sign) {
                if constexpr (IN) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float(&v)[VEC] = h ? b : a;
                        const int at = (h ? vb[i] : va[i]) * VEC;
                        if (at < 0 || at >= p.rotary) continue;
#pragma unroll
                        for (int m = 0; m + 1 < VEC; m += 2) {
                            const float2 cs = tw[(at + m) / 2];
                            const float s = sign * cs.y, u = v[m], w = v[m + 1];
                            v[m] = u * cs.x - w * s;
                            v[m + 1] = w * cs.x + u * s;
                        }
                    }
                } else {
                    const int u = lane + i * p.group;
                    if (u < p.hc) {
#pragma unroll
                        for (int m = 0; m < VEC; ++m) {
                            const float2 cs = tw[u * VEC + m];
                            const float s = sign * cs.y, q = a[m], w = b[m];
                            a[m] = q * cs.x - w * s;
                            b[m] = w * cs.x + q * s;
                        }
                    }
                }
            };
            float ss = 0.f, gx = 0.f;
            float fa[UPL][VEC], fb[UPL][VEC], da[BWD ? UPL : 1][VEC], db[BWD ? UPL : 1][VEC];
#pragma unroll
            for (int i = 0; i < UPL; ++i) {
                seq_unpack<T, VEC>(xa[i], fa[i]);
                seq_unpack<T, VEC>(xb[i], fb[i]);
#pragma unroll
                for (int m = 0; m < VEC; ++m) ss += fa[i][m] * fa[i][m] + fb[i][m] * fb[i][m];
                if constexpr (BWD) {
                    seq_unpack<T, VEC>(ya[i], da[i]);
                    seq_unpack<T, VEC>(yb[i], db[i]);
                    rotate(i, da[i], db[i], -1.f);
#pragma unroll
                    for (int m = 0; m < VEC; ++m) {
                        const float wa = va[i] >= 0 ? weight[va[i] * VEC + m] : 0.f, wb = vb[i] >= 0 ? weight[vb[i] * VEC + m] : 0.f;
                        gx += da[i][m] * wa * fa[i][m] + db[i][m] * wb * fb[i][m];
                    }
                }
            }
            for (int o = p.group / 2; o > 0; o >>= 1) {
                ss += __shfl_xor_sync(~0u, ss, o);
                if constexpr (BWD) gx += __shfl_xor_sync(~0u, gx, o);
            }
            const float rs = 1.f / sqrtf(ss * inv_d + p.eps);
            const float back = BWD ? rs * rs * (gx * inv_d) : 0.f;
#pragma unroll
            for (int i = 0; i < UPL; ++i) {
                if constexpr (BWD) {
                    if (sums && on) {
#pragma unroll
                        for (int m = 0; m < VEC; ++m) {
                            dwa[i][m] += da[i][m] * (fa[i][m] * rs);
                            dwb[i][m] += db[i][m] * (fb[i][m] * rs);
                        }
                    }
#pragma unroll
                    for (int m = 0; m < VEC; ++m) {
                        const float wa = va[i] >= 0 ? weight[va[i] * VEC + m] : 0.f, wb = vb[i] >= 0 ? weight[vb[i] * VEC + m] : 0.f;
                        fa[i][m] = rs * (da[i][m] * wa - fa[i][m] * back);
                        fb[i][m] = rs * (db[i][m] * wb - fb[i][m] * back);
                    }
                } else {
#pragma unroll
                    for (int m = 0; m < VEC; ++m) {
                        const float wa = va[i] >= 0 ? weight[va[i] * VEC + m] : 0.f, wb = vb[i] >= 0 ? weight[vb[i] * VEC + m] : 0.f;
                        fa[i][m] = fa[i][m] * rs * wa;
                        fb[i][m] = fb[i][m] * rs * wb;
                    }
                    rotate(i, fa[i], fb[i], 1.f);
                }
                if (on && va[i] >= 0) seq_store<T, VEC>(out + va[i] * VEC, seq_pack<T, VEC>(fa[i]));
                if (on && vb[i] >= 0) seq_store<T, VEC>(out + vb[i] * VEC, seq_pack<T, VEC>(fb[i]));
            }
        }
    }
    if constexpr (BWD) {
        if (!sums) return;
        // the row groups' sums, added in their order
        __syncthreads();
        float *acc = weight;  // [rows_at_once][D] would not fit for all: one group after another adds its own
        for (int j = threadIdx.x; j < p.D; j += kThreads) acc[j] = 0.f;
        for (int g = 0; g < rows_at_once; ++g) {
            __syncthreads();
            if (row0 != g) continue;
#pragma unroll
            for (int i = 0; i < UPL; ++i)
#pragma unroll
                for (int m = 0; m < VEC; ++m) {
                    if (va[i] >= 0) acc[va[i] * VEC + m] += dwa[i][m];
                    if (vb[i] >= 0) acc[vb[i] * VEC + m] += dwb[i][m];
                }
        }
        __syncthreads();
        for (int j = threadIdx.x; j < p.D; j += kThreads) sd.part[(long long)cta * p.D + j] = acc[j];
    }
}

// dweight[j] = sum of the CTAs' parts, 32 columns a block and 8 stretches of CTAs.
__global__ void __launch_bounds__(256) heads_weight_kernel(const float *part0, const float *part1, int ctas0, int ctas1, int D,
                                                           float *dw0, float *dw1) {
    __shared__ float sum[8][32];
    const bool keys = blockIdx.y;
    const float *part = keys ? part1 : part0;
    float *dw = keys ? dw1 : dw0;
    const int ctas = keys ? ctas1 : ctas0, x = threadIdx.x & 31, y = threadIdx.x >> 5, j = blockIdx.x * 32 + x;
    if (!dw) return;
    float v = 0.f;
    if (j < D)
        for (int c = y; c < ctas; c += 8) v += part[(long long)c * D + j];
    sum[y][x] = v;
    __syncthreads();
    if (y == 0 && j < D) {
        for (int k = 1; k < 8; ++k) v += sum[k][x];
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

// CTAs of queries and keys: 4 an SM over both, by their heads, no more than there are tiles.
void ctas_of(const wm_seq *h, const seq_heads_args &a, long long tiles, int (&ctas)[2]) {
    const int all = a.heads[0] + a.heads[1], room = 8 * h->sms;
    for (int i = 0; i < 2; ++i) {
        const long long share = a.heads[i] ? std::max(1ll, (long long)room * a.heads[i] / all) : 0;
        ctas[i] = (int)std::min(share, std::max(a.heads[i] ? 1ll : 0, tiles));
    }
}

int tile_of(const wm_seq *h, const seq_heads_args &a) {
    const long long tokens = a.T * a.N;
    // about an angle a thread, and no fewer tiles than CTAs
    const long long want = a.rotary ? std::max(1, 512 / a.rotary) : 16, fair = tokens / (8ll * h->sms);
    return (int)std::max(1ll, std::min({want, fair, 16ll}));
}

template <class T, int VEC, bool IN, int UPL>
cudaError_t run(wm_seq *h, const HeadArgs &p, bool backward, cudaStream_t s) {
    const size_t bytes = (size_t)p.rotary / 2 * 8 * (1 + p.tile) + (size_t)((p.D + VEC - 1) / VEC * VEC) * 4;
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
cudaError_t run_units(wm_seq *h, HeadArgs &p, bool backward, cudaStream_t s) {
    int g = 1;
    while (g < 32 && g < p.units) g <<= 1;
    p.group = g;
    const int upl = (p.units + g - 1) / g;
    if (upl <= 1) return run<T, VEC, IN, 1>(h, p, backward, s);
    if constexpr (VEC <= 4 || sizeof(T) == 2) {
        if (upl <= 2) return run<T, VEC, IN, 2>(h, p, backward, s);
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
        if (vec == 8) return in ? run_units<T, 8, true>(h, p, backward, s) : run_units<T, 8, false>(h, p, backward, s);
    }
    if (vec == 4) return in ? run_units<T, 4, true>(h, p, backward, s) : run_units<T, 4, false>(h, p, backward, s);
    if (vec == 2) return in ? run_units<T, 2, true>(h, p, backward, s) : run_units<T, 2, false>(h, p, backward, s);
    return run_units<T, 1, false>(h, p, backward, s);
}

}  // namespace

size_t wm_seq_heads_backward_ws(const wm_seq *h, const seq_heads_args &a) {
    if (!a.dweight[0] && !a.dweight[1]) return 0;
    int ctas[2];
    const int tile = tile_of(h, a);
    ctas_of(h, a, (a.T * a.N + tile - 1) / tile, ctas);
    return (size_t)(ctas[0] + ctas[1]) * a.D * 4;
}

cudaError_t wm_seq_heads_launch(wm_seq *h, const seq_heads_args &a, bool backward, cudaStream_t s) {
    h->last_launches = 0;
    HeadArgs p{};
    p.tokens = a.T * a.N;
    p.N = a.N; p.D = a.D; p.rotary = a.rotary; p.eps = a.eps;
    p.positions = a.positions; p.freqs = a.freqs;
    p.tile = tile_of(h, a);
    int ctas[2];
    ctas_of(h, a, (p.tokens + p.tile - 1) / p.tile, ctas);
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
    heads_weight_kernel<<<dim3((a.D + 31) / 32, 2), 256, 0, s>>>(p.side[0].part, p.side[1].part, ctas[0], ctas[1], a.D, a.dweight[0],
                                                                 a.dweight[1]);
    return cudaGetLastError();
}
