// libpgf: preparation of queries and keys (norm per head, weight, rotation by
// position) and its adjoint, for gfx950.
//
// Per head and step  y = R (w * x r), r = (c sum x^2 + eps)^-1/2.  With the
// adjoint signal dy: du = R^T dy, dw = sum of du * x r over steps and heads,
// and, t = du * w,  dx = r (t - c r^2 x (x . t)).
//
// One pass: a group of G = 2^n >= d / 8 lanes holds one head vector, eight
// elements a lane (16 bytes of bf16), sums by DPP and lane swaps.  The two halves of a
// rotated pair lie in one lane (interleaved) or in lanes rot / 16 apart.  A
// block takes a few steps and all their heads, so each angle is computed once
// per step, not per head: the turn position * inv_freq / 2 pi in f64, reduced
// to [-1/2, 1/2] there, then sine and cosine in f32.
#include "pgf_gdr.h"
#include "pgf_timing.h"

namespace pgf {
namespace qk {

using gdr::View;
using gdr::floatx4;
using gdr::bf16x8;

struct Args {
    View x[2], y[2], dy[2];          // q and k
    const float *w[2];
    const float *inv_freq;
    const void *pos;
    int64_t pos_stride;
    int pos64, d, rot, il, l2;
    int64_t L, rows;                 // rows: batch entries * steps
    int H0, H;                       // query heads, all heads
    float eps, c;                    // c = 0: no norm
    int tb;                          // steps per block and turn
    float *part;                     // [blocks][2][d] partial sums of dw
};

template <typename T>
__device__ __forceinline__ void load8(const T *p, float (&v)[8]) {
    if constexpr (sizeof(T) == 2) {
        const bf16x8 x = *(const bf16x8 *)p;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)x[i];
    } else {
        const floatx4 a = ((const floatx4 *)p)[0], b = ((const floatx4 *)p)[1];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i] = a[i];
            v[4 + i] = b[i];
        }
    }
}
template <typename T>
__device__ __forceinline__ void store8(T *p, const float (&v)[8]) {
    if constexpr (sizeof(T) == 2) {
        bf16x8 x;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (__bf16)v[i];
        *(bf16x8 *)p = x;
    } else {
        ((floatx4 *)p)[0] = floatx4{v[0], v[1], v[2], v[3]};
        ((floatx4 *)p)[1] = floatx4{v[4], v[5], v[6], v[7]};
    }
}

// Sum over a group of G lanes, in every lane of it.
template <int G>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
    for (int m = 1; m < G; m *= 2) v += __shfl_xor(v, m, 64);
    return v;
}

constexpr int kPairs = 256;          // rotated pairs of a step at most
constexpr int kTurn = 8;             // steps per block and turn at most

// Rotation of a lane's eight elements (sgn = -1: back).  cs: cosine and sine
// of the step's pairs.
template <int G>
__device__ __forceinline__ void rotate(float (&v)[8], const float2 *cs, int e0, int rot, int il, float sgn) {
    if (il) {
        if (e0 < rot) {
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                const float2 t = cs[(e0 + i) / 2];
                const float a = v[i], b = v[i + 1], s = sgn * t.y;
                v[i] = a * t.x - b * s;
                v[i + 1] = b * t.x + a * s;
            }
        }
        return;
    }
    const int half = rot / 2, hl = half / 8;       // lanes from one element of a pair to the other
    const int lane = threadIdx.x % 64;
    const bool first = e0 < half, in = e0 < rot;
    const int other = in ? (first ? lane + hl : lane - hl) : lane;
    const int at = in ? (first ? e0 : e0 - half) : 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float o = __shfl(v[i], other, 64);
        if (in) {
            const float2 t = cs[at + i];
            const float s = (first ? -sgn : sgn) * t.y;
            v[i] = v[i] * t.x + o * s;
        }
    }
}

// Bound by memory: x is read and y written once (and dy read by the adjoint).
template <typename T, int G, bool GRAD>
__global__ __launch_bounds__(256) void k_qk(Args a) {
    __shared__ float2 sCs[kTurn * kPairs];
    __shared__ float sW[GRAD ? 2 * 512 : 1];
    __shared__ int64_t sBT[kTurn][2];              // batch entry and step
    constexpr int NG = 256 / G;                    // head vectors at a time
    const int tid = threadIdx.x, grp = tid / G, e0 = tid % G * 8;
    const bool on = e0 < a.d;
    const int half = a.rot / 2;
    float w[2][8], dw[2][8];
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            w[x][i] = a.w[x] && on ? a.w[x][e0 + i] : 1.0f;
            dw[x][i] = 0.0f;
        }
    for (int64_t r0 = (int64_t)blockIdx.x * a.tb; r0 < a.rows; r0 += (int64_t)gridDim.x * a.tb) {
        const int nt = (int)(a.rows - r0 < a.tb ? a.rows - r0 : a.tb);
        __syncthreads();
        if (tid < nt) {
            sBT[tid][0] = (r0 + tid) / a.L;
            sBT[tid][1] = (r0 + tid) - sBT[tid][0] * a.L;
        }
        __syncthreads();
        if (a.rot) {
            for (int i = tid; i < nt * half; i += 256) {
                const int64_t b = sBT[i / half][0], t = sBT[i / half][1];
                const int64_t at = b * a.pos_stride + t;
                const double pos = !a.pos ? (double)t : a.pos64 ? (double)((const int64_t *)a.pos)[at]
                                                                : (double)((const int32_t *)a.pos)[at];
                double turns = pos * (double)a.inv_freq[i % half] * 0.15915494309189533577;   // 1 / 2 pi
                turns -= rint(turns);
                float s, c;
                sincospif(2.0f * (float)turns, &s, &c);
                sCs[i] = float2{c, s};
            }
            __syncthreads();
        }
        const int units = nt * a.H;
        for (int u0 = 0; u0 < units; u0 += NG) {
            const int u = u0 + grp;
            const bool live = u < units;           // lanes of one group agree
            const int s = live ? u / a.H : 0, hh = live ? u - s * a.H : 0;
            const int x = hh >= a.H0;              // 0 = query, 1 = key
            const int h = x ? hh - a.H0 : hh;
            const int64_t b = sBT[s][0], t = sBT[s][1];
            const bool act = live && on;
            float v[8] = {};
            if (act) load8((x ? a.x[1] : a.x[0]).template at<const T>(b, h, t) + e0, v);
            float ss = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) ss = fmaf(v[i], v[i], ss);
            ss = group_sum<G>(ss);
            const float rs = a.c == 0.0f ? 1.0f : 1.0f / sqrtf(fmaf(ss, a.c, a.eps));
            const float2 *cs = sCs + s * half;
            if constexpr (!GRAD) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = v[i] * rs * (x ? w[1][i] : w[0][i]);
                if (a.rot) rotate<G>(v, cs, e0, a.rot, a.il, 1.0f);
                if (act) store8((x ? a.y[1] : a.y[0]).template at<T>(b, h, t) + e0, v);
            } else {
                float g[8] = {};
                if (act) load8((x ? a.dy[1] : a.dy[0]).template at<const T>(b, h, t) + e0, g);
                if (a.rot) rotate<G>(g, cs, e0, a.rot, a.il, -1.0f);
                float dot = 0.0f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float xr = g[i] * (v[i] * rs);
                    if (live) {
                        dw[0][i] += x ? 0.0f : xr;
                        dw[1][i] += x ? xr : 0.0f;
                    }
                    g[i] *= x ? w[1][i] : w[0][i];
                    dot = fmaf(v[i], g[i], dot);
                }
                dot = group_sum<G>(dot) * (rs * rs * a.c);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = rs * (g[i] - v[i] * dot);
                if (act) store8((x ? a.y[1] : a.y[0]).template at<T>(b, h, t) + e0, v);
            }
        }
    }
    if constexpr (GRAD) {
        if (!a.part) return;
        // The groups' sums in order: a wave's by lane exchange, the waves' one after the other.
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float v = dw[x][i];
#pragma unroll
                for (int m = G; m < 64; m *= 2) v += __shfl_xor(v, m, 64);
                dw[x][i] = v;
            }
        for (int wv = 0; wv < 4; ++wv) {
            if (tid / 64 == wv && tid % 64 < G && on) {
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        float &s = sW[x * 512 + e0 + i];
                        s = wv ? s + dw[x][i] : dw[x][i];
                    }
            }
            __syncthreads();
        }
        for (int i = tid; i < 2 * a.d; i += 256) {
            const int x = i >= a.d;
            a.part[(int64_t)blockIdx.x * 2 * a.d + i] = sW[x * 512 + i - x * a.d];
        }
    }
}

// dw of one element of the query's (x = 0) or key's weight: the blocks'
// partial sums, a fixed share per lane, then over the lanes.
__global__ __launch_bounds__(64) void k_qk_dw(const float *part, int blocks, int d, float *dwq, float *dwk) {
    const int e = blockIdx.x, x = e >= d;
    float *out = x ? dwk : dwq;
    if (!out) return;
    float s = 0.0f;
    for (int b = threadIdx.x; b < blocks; b += 64) s += part[(int64_t)b * 2 * d + e];
#pragma unroll
    for (int m = 1; m < 64; m *= 2) s += __shfl_xor(s, m, 64);
    if (threadIdx.x == 0) out[x ? e - d : e] = s;
}

View view(const void *p, const int64_t (&s)[3], int64_t H, int64_t L, int64_t d) {
    int64_t o[3];
    dense_strides(s, H, L, d, o);
    return View{p, o[0], o[1], o[2]};
}

template <typename T, bool GRAD>
void launch(const Args &a, int G, unsigned blocks, hipStream_t st) {
    switch (G) {
        case 1: hipLaunchKernelGGL((k_qk<T, 1, GRAD>), dim3(blocks), dim3(256), 0, st, a); break;
        case 2: hipLaunchKernelGGL((k_qk<T, 2, GRAD>), dim3(blocks), dim3(256), 0, st, a); break;
        case 4: hipLaunchKernelGGL((k_qk<T, 4, GRAD>), dim3(blocks), dim3(256), 0, st, a); break;
        case 8: hipLaunchKernelGGL((k_qk<T, 8, GRAD>), dim3(blocks), dim3(256), 0, st, a); break;
        case 16: hipLaunchKernelGGL((k_qk<T, 16, GRAD>), dim3(blocks), dim3(256), 0, st, a); break;
        case 32: hipLaunchKernelGGL((k_qk<T, 32, GRAD>), dim3(blocks), dim3(256), 0, st, a); break;
        default: hipLaunchKernelGGL((k_qk<T, 64, GRAD>), dim3(blocks), dim3(256), 0, st, a); break;
    }
}

int run(const void *q, const void *k, const void *dq, const void *dk, const pgf_qk_params *p, void *qo, void *ko,
        void *stream, bool grads) {
    Plan pl;
    const int rc = make_plan(p, &pl, grads);
    if (rc != PGF_OK) return rc;
    if (grads && ((p->w_q && pl.Hq && !p->grad_w_q) || (p->w_k && pl.Hk && !p->grad_w_k))) return PGF_ERR_INVALID_ARG;
    if (grads && pl.total && (!p->workspace || p->workspace_bytes < pl.total || ((uintptr_t)p->workspace & 255)))
        return PGF_ERR_WORKSPACE;
    const size_t e = p->in_dtype == PGF_BF16 ? 2 : 4;
    const bool some = pl.L > 0;
    const struct { const void *x, *dy; void *y; const int64_t (&xs)[3], (&ds)[3], (&ys)[3]; int64_t H; } sides[2] = {
        {q, dq, qo, p->q_strides, p->dq_strides, p->q_out_strides, pl.Hq},
        {k, dk, ko, p->k_strides, p->dk_strides, p->k_out_strides, pl.Hk}};
    if (some) {
        for (const auto &s : sides) {
            if (!s.H) continue;
            if (!s.x || !s.y || (grads && !s.dy)) return PGF_ERR_INVALID_ARG;
            if (((uintptr_t)s.x | (uintptr_t)s.y | (grads ? (uintptr_t)s.dy : 0)) & 15) return PGF_ERR_INVALID_ARG;
        }
        for (const auto &o : sides) {
            if (!o.H) continue;
            const size_t ny = extent(o.ys, pl.B, o.H, pl.L, pl.d, e);
            int64_t oy[3], ix[3];
            dense_strides(o.ys, o.H, pl.L, pl.d, oy);
            for (const auto &s : sides) {
                if (!s.H) continue;
                // An output over an input: only itself, element on element.
                const struct { const void *p; const int64_t (&st)[3]; } ins[2] = {{s.x, s.xs}, {grads ? s.dy : nullptr, s.ds}};
                for (const auto &in : ins) {
                    if (!overlaps(o.y, ny, in.p, extent(in.st, pl.B, s.H, pl.L, pl.d, e))) continue;
                    dense_strides(in.st, s.H, pl.L, pl.d, ix);
                    const bool same = in.p == o.y && &s == &o && ix[0] == oy[0] && ix[1] == oy[1] && ix[2] == oy[2];
                    // Heads of one fused array: the other side's rows interleave with these.
                    const bool apart = &s != &o && ix[0] == oy[0] && ix[2] == oy[2];
                    if (!same && !apart) return PGF_ERR_INVALID_ARG;
                }
            }
            if (overlaps(o.y, ny, p->workspace, pl.total)) return PGF_ERR_INVALID_ARG;
        }
    }
    (void)hipGetLastError();
    hipStream_t st = (hipStream_t)stream;
    Args a{};
    for (int x = 0; x < 2; ++x) {
        const auto &s = sides[x];
        a.x[x] = view(s.x, s.xs, s.H, pl.L, pl.d);
        a.y[x] = view(s.y, s.ys, s.H, pl.L, pl.d);
        a.dy[x] = view(s.dy, s.ds, s.H, pl.L, pl.d);
    }
    a.w[0] = p->w_q;
    a.w[1] = p->w_k;
    a.inv_freq = p->inv_freq;
    a.pos = p->positions;
    a.pos_stride = p->pos_stride;
    a.pos64 = p->pos_bits == 64;
    a.d = (int)pl.d;
    a.rot = (int)pl.rot;
    a.il = p->interleaved != 0;
    a.L = some ? pl.L : 1;
    a.rows = pl.B * pl.L;
    a.H0 = (int)pl.Hq;
    a.H = (int)(pl.Hq + pl.Hk);
    a.eps = p->eps;
    a.c = p->norm == PGF_NORM_NONE ? 0.0f : p->norm == PGF_NORM_L2 ? 1.0f : 1.0f / (float)pl.d;
    // Steps per block: one while that leaves the GPU idle, then as many as fill
    // a few turns of the block's head groups.
    const int64_t per = 256 / pl.G;
    a.tb = 1;
    while (a.tb < kTurn && a.tb * a.H < 4 * per && a.rows / (2 * a.tb) >= 1024) a.tb *= 2;
    const int64_t want = (a.rows + a.tb - 1) / a.tb;
    const bool bf = p->in_dtype == PGF_BF16;
    if (!grads) {
        if (a.rows == 0) return PGF_OK;
        Timed tm(0, st);
        if (bf) launch<__bf16, false>(a, pl.G, (unsigned)want, st);
        else launch<float, false>(a, pl.G, (unsigned)want, st);
    } else {
        a.part = pl.total ? (float *)p->workspace : nullptr;
        const unsigned blocks = (unsigned)(want < pl.blocks ? (want > 0 ? want : 1) : pl.blocks);
        {
            Timed tm(3, st);
            if (bf) launch<__bf16, true>(a, pl.G, blocks, st);
            else launch<float, true>(a, pl.G, blocks, st);
        }
        if (a.part) {
            Timed tm(2, st);
            hipLaunchKernelGGL(k_qk_dw, dim3((unsigned)(2 * pl.d)), dim3(64), 0, st, (const float *)a.part, (int)blocks,
                               (int)pl.d, p->w_q ? p->grad_w_q : nullptr, p->w_k ? p->grad_w_k : nullptr);
        }
    }
    return hipGetLastError() == hipSuccess ? PGF_OK : PGF_ERR_HIP;
}

}  // namespace qk
}  // namespace pgf

extern "C" int pgf_qk_norm(const void *q, const void *k, const pgf_qk_params *p, void *q_out, void *k_out, void *stream) {
    return pgf::qk::run(q, k, nullptr, nullptr, p, q_out, k_out, stream, false);
}

extern "C" int pgf_qk_norm_grads(const void *q, const void *k, const void *dq, const void *dk, const pgf_qk_params *p,
                                 void *q_out, void *k_out, void *stream) {
    return pgf::qk::run(q, k, dq, dk, p, q_out, k_out, stream, true);
}
