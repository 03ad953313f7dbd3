// libpgf: preparation of queries and keys (norm per head, weight, rotation by
// position) and its adjoint, for gfx950.
//
// Per head and step  y = R (w * x r), r = (c sum x^2 + eps)^-1/2.  With the
// adjoint signal dy: du = R^T dy, dw = sum of du * x r over steps and heads,
// and, t = du * w,  dx = r (t - c r^2 x (x . t)).
//
// One pass: a group of G = 2^n >= d / 8 lanes holds one head vector, eight
// elements a lane in two runs of four.  In the rotated part of a vector whose
// pairs are (i, i + rot / 2) a lane's runs are the two halves of the same four
// pairs, elsewhere they follow each other, so a rotation never leaves the lane
// and reads four cosines and sines.  Sums go by DPP.  A block takes a few steps
// and all their heads, so each angle is computed once per step, not per head: the
// turn position * inv_freq / 2 pi, reduced to [-1/2, 1/2], and its sine and cosine
// in f64, rounded to f32 once.
#include "pgf_gdr.h"
#include "pgf_timing.h"

namespace pgf {
namespace qk {

using gdr::View;
using gdr::floatx4;

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

using gdr::Raw4;
using gdr::load4;

// Sum over a group of G lanes, in every lane of it.
template <int CTRL>
__device__ __forceinline__ float add_dpp(float v) {
    return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, false));
}
template <int G>
__device__ __forceinline__ float group_sum(float v) {
    if constexpr (G > 1) v = add_dpp<0xB1>(v);     // lane ^ 1
    if constexpr (G > 2) v = add_dpp<0x4E>(v);     // lane ^ 2: sums of quads
    if constexpr (G > 4) v = add_dpp<0x141>(v);    // 7 - lane: the other quad's
    if constexpr (G > 8) v = add_dpp<0x140>(v);    // 15 - lane: the other eight's
#pragma unroll
    for (int m = 16; m < G; m *= 2) v += __shfl_xor(v, m, 64);
    return v;
}

constexpr int kPairs = 256;          // rotated pairs of a step at most

// Cosine and sine of `turns` in [-1/2, 1/2], in f64 and rounded once: the nearest
// quarter is taken off, exactly, and the series of the rest, at most pi / 4, leave
// 2^-52 at the terms x^15 and x^16.  (The library's sincospi takes the adjoint more
// registers than it has: 108 us in place of 103 for 4 x 4096 steps of 32 heads.)
__device__ __forceinline__ float2 cos_sin(double turns) {
    const double n = rint(4.0 * turns);
    const double x = 6.28318530717958647693 * fma(-0.25, n, turns), z = x * x;
    constexpr double f3 = 6, f5 = 120, f7 = 5040, f9 = 362880, f11 = 39916800, f13 = 6227020800.0, f15 = 1307674368000.0;
    double s = -1.0 / f15;
    s = fma(s, z, 1.0 / f13);
    s = fma(s, z, -1.0 / f11);
    s = fma(s, z, 1.0 / f9);
    s = fma(s, z, -1.0 / f7);
    s = fma(s, z, 1.0 / f5);
    s = fma(s, z, -1.0 / f3);
    const float sn = (float)fma(s * z, x, x);
    double c = 1.0 / (f15 * 16);
    c = fma(c, z, -1.0 / (f13 * 14));
    c = fma(c, z, 1.0 / (f11 * 12));
    c = fma(c, z, -1.0 / (f9 * 10));
    c = fma(c, z, 1.0 / (f7 * 8));
    c = fma(c, z, -1.0 / (f5 * 6));
    c = fma(c, z, 1.0 / (f3 * 4));
    c = fma(c, z, -0.5);
    const float cn = (float)fma(c, z, 1.0);
    const int k = (int)n & 3;            // quarters
    const float a = k & 1 ? sn : cn, b = k & 1 ? cn : sn;
    return float2{k == 1 || k == 2 ? -a : a, k >= 2 ? -b : b};
}

// Rotation of a lane's runs (sgn = -1: back); cs: of its four pairs.
__device__ __forceinline__ void rotate(floatx4 &x, floatx4 &y, const float2 *cs, int il, float sgn) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float c = cs[i].x, s = sgn * cs[i].y;
        if (il) {                    // pairs (x0, x1), (x2, x3), (y0, y1), (y2, y3)
            floatx4 &v = i < 2 ? x : y;
            const float a = v[2 * (i & 1)], b = v[2 * (i & 1) + 1];
            v[2 * (i & 1)] = a * c - b * s;
            v[2 * (i & 1) + 1] = b * c + a * s;
        } else {                     // pairs (x_i, y_i)
            const float a = x[i], b = y[i];
            x[i] = a * c - b * s;
            y[i] = b * c + a * s;
        }
    }
}

template <typename T>
__device__ __forceinline__ void store4(T *p, const floatx4 &v) {
    Raw4<T> r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.x[i] = (T)v[i];
    *(Raw4<T> *)p = r;
}

// Bound by memory: x is read and y written once (and dy read by the adjoint):
// 16384 steps of 32 heads of 128 in bf16 72 us (3.7 TB/s), the adjoint 99 us (4.1; a
// few registers spill around the angles, 10 MB of 403, without which it takes as long).
// The next vector is loaded while one is computed, the first ones while the
// angles are.
template <typename T, int G, bool GRAD>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(4))) void k_qk(Args a) {
    __shared__ __align__(16) float2 sCs[kTurn * kPairs];
    __shared__ float sW[GRAD ? 2 * 512 : 1];
    __shared__ int64_t sBT[kTurn][2];              // batch entry and step
    constexpr int NG = 256 / G;                    // head vectors at a time
    const int tid = threadIdx.x, grp = tid / G, li = tid % G;
    const bool on = 8 * li < a.d, turned = 8 * li < a.rot;
    const int half = a.rot / 2;
    // the lane's runs of elements, and its pairs
    const int e0 = turned && !a.il ? 4 * li : 8 * li, e1 = turned && !a.il ? half + 4 * li : 8 * li + 4;
    floatx4 w[2][2], dw[2][2];
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[x][0][i] = a.w[x] && on ? a.w[x][e0 + i] : 1.0f;
            w[x][1][i] = a.w[x] && on ? a.w[x][e1 + i] : 1.0f;
            dw[x][0][i] = dw[x][1][i] = 0.0f;
        }
    struct Unit {
        Raw4<T> x[2], g[GRAD ? 2 : 1];
    };
    for (int64_t r0 = (int64_t)blockIdx.x * a.tb; r0 < a.rows; r0 += (int64_t)gridDim.x * a.tb) {
        const int nt = (int)(a.rows - r0 < a.tb ? a.rows - r0 : a.tb);
        const int units = nt * a.H;
        __syncthreads();
        if (tid < nt) {
            sBT[tid][0] = (r0 + tid) / a.L;
            sBT[tid][1] = (r0 + tid) - sBT[tid][0] * a.L;
        }
        __syncthreads();
        // place of unit u (a lane without one repeats the last, and does not store)
        int s, x, h;
        int64_t b, t;
        auto place = [&](int u) {
            u = u < units ? u : units - 1;
            s = u / a.H;
            h = u - s * a.H;
            x = h >= a.H0;                         // 0 = query, 1 = key
            h -= x ? a.H0 : 0;
            b = sBT[s][0];
            t = sBT[s][1];
        };
        auto fetch = [&](int u) {
            place(u);
            Unit v;
            const T *p = (x ? a.x[1] : a.x[0]).template at<const T>(b, h, t);
            const int f0 = on ? e0 : 0, f1 = on ? e1 : 0;
            v.x[0] = load4(p + f0);
            v.x[1] = load4(p + f1);
            if constexpr (GRAD) {
                const T *q = (x ? a.dy[1] : a.dy[0]).template at<const T>(b, h, t);
                v.g[0] = load4(q + f0);
                v.g[1] = load4(q + f1);
            }
            return v;
        };
        Unit next = fetch(grp);
        if (a.rot) {
            for (int i = tid; i < nt * half; i += 256) {
                const int64_t at = sBT[i / half][0] * a.pos_stride + sBT[i / half][1];
                const double pos = !a.pos ? (double)sBT[i / half][1] : a.pos64 ? (double)((const int64_t *)a.pos)[at]
                                                                               : (double)((const int32_t *)a.pos)[at];
                double turns = pos * (double)a.inv_freq[i % half] * 0.15915494309189533577;   // 1 / 2 pi
                turns -= rint(turns);
                sCs[i] = cos_sin(turns);
            }
            __syncthreads();
        }
        for (int u0 = 0; u0 < units; u0 += NG) {
            const Unit cur = next;
            next = fetch(u0 + NG + grp);
            place(u0 + grp);
            const bool live = u0 + grp < units, act = live && on;      // lanes of one group agree on live
            floatx4 v0 = cur.x[0].f(), v1 = cur.x[1].f();
            float ss = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) ss = fmaf(v0[i], v0[i], fmaf(v1[i], v1[i], ss));
            ss = group_sum<G>(on ? ss : 0.0f);
            const float rs = a.c == 0.0f ? 1.0f : 1.0f / sqrtf(fmaf(ss, a.c, a.eps));
            const float2 *cs = sCs + s * half + 4 * li;
            T *out = (x ? a.y[1] : a.y[0]).template at<T>(b, h, t);
            const floatx4 w0 = x ? w[1][0] : w[0][0], w1 = x ? w[1][1] : w[0][1];
            if constexpr (!GRAD) {
                v0 = v0 * rs * w0;
                v1 = v1 * rs * w1;
                if (turned) rotate(v0, v1, cs, a.il, 1.0f);
            } else {
                floatx4 g0 = cur.g[0].f(), g1 = cur.g[1].f();
                if (turned) rotate(g0, g1, cs, a.il, -1.0f);
                const floatx4 d0 = g0 * (v0 * rs), d1 = g1 * (v1 * rs);
                if (live) {
                    if (x) {
                        dw[1][0] += d0;
                        dw[1][1] += d1;
                    } else {
                        dw[0][0] += d0;
                        dw[0][1] += d1;
                    }
                }
                g0 *= w0;
                g1 *= w1;
                float dot = 0.0f;
#pragma unroll
                for (int i = 0; i < 4; ++i) dot = fmaf(v0[i], g0[i], fmaf(v1[i], g1[i], dot));
                dot = group_sum<G>(on ? dot : 0.0f) * (rs * rs * a.c);
                v0 = rs * (g0 - v0 * dot);
                v1 = rs * (g1 - v1 * dot);
            }
            if (act) {
                store4(out + e0, v0);
                store4(out + e1, v1);
            }
        }
    }
    if constexpr (GRAD) {
        if (!a.part) return;
        // The groups' sums in order: a wave's by lane exchange, the waves' one after the other.
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float v = dw[x][k][i];
#pragma unroll
                    for (int m = G; m < 64; m *= 2) v += __shfl_xor(v, m, 64);
                    dw[x][k][i] = v;
                }
        for (int wv = 0; wv < 4; ++wv) {
            if (tid / 64 == wv && tid % 64 < G && on) {
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float &s0 = sW[x * 512 + e0 + i], &s1 = sW[x * 512 + e1 + i];
                        s0 = wv ? s0 + dw[x][0][i] : dw[x][0][i];
                        s1 = wv ? s1 + dw[x][1][i] : dw[x][1][i];
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

// dw of 32 elements (the query's weight, then the key's): 32 threads an element
// sum a fixed share of the blocks' partial sums each, and then each other's.
__global__ __launch_bounds__(1024) void k_qk_dw(const float *part, int blocks, int d, float *dwq, float *dwk) {
    __shared__ float sS[32][33];
    const int c = threadIdx.x % 32, g = threadIdx.x / 32;
    const int e = blockIdx.x * 32 + c;
    float s = 0.0f;
    if (e < 2 * d) {
#pragma unroll 4
        for (int b = g; b < blocks; b += 32) s += part[(int64_t)b * 2 * d + e];
    }
    sS[g][c] = s;
    __syncthreads();
    s = sS[c][g];                                  // element g of the 32, share c
#pragma unroll
    for (int m = 1; m < 32; m *= 2) s += __shfl_xor(s, m, 32);
    const int o = blockIdx.x * 32 + g, x = o >= d;
    float *out = x ? dwk : dwq;
    if (c == 0 && o < 2 * d && out) out[x ? o - d : o] = s;
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
    if (((uintptr_t)p->w_q | (uintptr_t)p->w_k | (uintptr_t)p->inv_freq |
         (grads ? (uintptr_t)p->grad_w_q | (uintptr_t)p->grad_w_k : 0)) & 3)
        return PGF_ERR_INVALID_ARG;
    if (pl.rot && p->positions && (uintptr_t)p->positions % (size_t)(p->pos_bits / 8)) return PGF_ERR_INVALID_ARG;
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
        const Arr outs[2] = {{qo, p->q_out_strides, pl.B, pl.Hq, pl.L, pl.d, e}, {ko, p->k_out_strides, pl.B, pl.Hk, pl.L, pl.d, e}};
        const Arr ins[4] = {{q, p->q_strides, pl.B, pl.Hq, pl.L, pl.d, e}, {k, p->k_strides, pl.B, pl.Hk, pl.L, pl.d, e},
                            {grads ? dq : nullptr, p->dq_strides, pl.B, pl.Hq, pl.L, pl.d, e},
                            {grads ? dk : nullptr, p->dk_strides, pl.B, pl.Hk, pl.L, pl.d, e}};
        for (int i = 0; i < 2; ++i) {
            for (int j = 0; j < 4; ++j) {
                if (!overlaps(outs[i], ins[j])) continue;
                // An output over an input: only its own, element on element (an
                // index of one value has no stride to differ in).
                const int64_t n[3] = {pl.B, outs[i].H, pl.L};
                int64_t x[3], y[3];
                dense_strides(outs[i].s, outs[i].H, pl.L, pl.d, x);
                dense_strides(ins[j].s, ins[j].H, pl.L, pl.d, y);
                bool same = j % 2 == i && outs[i].p == ins[j].p;
                for (int e = 0; e < 3; ++e) same = same && (n[e] == 1 || x[e] == y[e]);
                if (!same) return PGF_ERR_INVALID_ARG;
            }
        }
        if (overlaps(outs[0], outs[1])) return PGF_ERR_INVALID_ARG;
        // The dense arrays: what is written (first the outputs, then the weights'
        // gradients and the workspace) lies apart from what is read and from each other.
        struct Range { const void *p; size_t n; };
        const size_t nw = (size_t)pl.d * 4, nf = (size_t)pl.rot / 2 * 4;
        const size_t np = pl.rot ? (size_t)((pl.B - 1) * p->pos_stride + pl.L) * (size_t)(p->pos_bits / 8) : 0;
        const Range written[] = {{outs[0].p, outs[0].bytes()}, {outs[1].p, outs[1].bytes()},
                                 {grads && p->w_q ? p->grad_w_q : nullptr, nw}, {grads && p->w_k ? p->grad_w_k : nullptr, nw},
                                 {grads ? p->workspace : nullptr, pl.total}};
        const Range read[] = {{p->w_q, nw}, {p->w_k, nw}, {p->inv_freq, nf}, {p->positions, np}};
        for (int i = 0; i < 5; ++i) {
            for (const auto &x : read)
                if (overlaps(written[i].p, written[i].n, x.p, x.n)) return PGF_ERR_INVALID_ARG;
            if (i < 2) continue;
            for (const auto &x : ins)
                if (overlaps(written[i].p, written[i].n, x.p, x.bytes())) return PGF_ERR_INVALID_ARG;
            for (int j = 0; j < i; ++j)
                if (overlaps(written[i].p, written[i].n, written[j].p, written[j].n)) return PGF_ERR_INVALID_ARG;
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
    a.tb = pl.tb;
    const bool bf = p->in_dtype == PGF_BF16;
    if (!grads) {
        if (a.rows == 0) return PGF_OK;
        Timed tm(0, st);
        if (bf) launch<__bf16, false>(a, pl.G, (unsigned)pl.blocks, st);
        else launch<float, false>(a, pl.G, (unsigned)pl.blocks, st);
    } else {
        a.part = pl.total ? (float *)p->workspace : nullptr;
        const unsigned blocks = (unsigned)pl.grad_blocks;
        {
            Timed tm(3, st);
            if (bf) launch<__bf16, true>(a, pl.G, blocks, st);
            else launch<float, true>(a, pl.G, blocks, st);
        }
        if (a.part) {
            Timed tm(2, st);
            hipLaunchKernelGGL(k_qk_dw, dim3((unsigned)((2 * pl.d + 31) / 32)), dim3(1024), 0, st, (const float *)a.part, (int)blocks,
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
