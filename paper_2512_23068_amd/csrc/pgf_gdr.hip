// libpgf: the gated delta rule for gfx950: scan over whole sequences and single
// steps on a pool of states.
//
// Chunk form (C = 32 steps; G the sum of g within the chunk up to and including
// a step, S the state entering it, N = tril(e^{G_t - G_s} * K K^T, -1),
// A = tril(e^{G_t - G_s} * Q K^T)): with E = V - (what S holds for the keys when
// their steps come), so that the steps write diag(beta) E,
//   X = V - e^G K S,   E = T^ X,   T^ = (I + N diag(beta))^-1
//   O = scale (e^G Q S + TA X),        TA = A diag(beta) T^
//   S' = e^{G_C} S + K^T (TW X),       TW = diag(e^{G_C - G} beta) T^
// T^, TA and TW depend on the chunk's keys and gates alone.
//
//   k_gdr_prep    per chunk and head: TW, TA (no dependence between chunks)
//   k_gdr_chain   per head and 16 value columns a wave: the chain over chunks
//   k_gdr_carry   composes segments of chunks where sequences are cut
//   k_gdr_step    single steps
//
// Why chunks of 32: a product with T^ is one contraction of the 16x16x32 matrix
// instruction, and a chunk's keys, queries, TW and TA take 26 KB of LDS in bf16,
// so that two blocks share a CU, each with the next chunk behind.
#include "pgf_gdr_chain.h"
#include "pgf_timing.h"

namespace pgf {
namespace gdr {

// ---------------------------------------------------------------- single steps
// A block holds CB value columns of one state in registers: thread (kg, cg)
// has the keys kg + KG i of the columns 4 cg .. 4 cg + 3.  One pass forms S^T k
// and S^T q on the decayed state together (o = S^T q + (k.q) u after the
// write), so a token costs one reduction over the block.  Bound by memory: the
// state is read and written once, whatever the number of steps (one step of 4096
// states of 128 x 128 88 us, 6.0 TB/s); a single state's step by latency (5 us).
template <typename T, int DK, int CB>
__global__ __launch_bounds__(256) void k_gdr_step(Args a, float *pool, int64_t n_pool, const int32_t *slots, int64_t L,
                                                  uint32_t n_items) {
    constexpr int CG = CB / 4, KG = 256 / CG, KPT = DK / KG;      // keys a thread
    __shared__ __align__(16) float sKQ[2][DK];
    __shared__ __align__(16) floatx4 sRed[4][2][CG];
    __shared__ float sDot[4];
    __shared__ int sDup;
    const int tid = threadIdx.x, cg = tid % CG, kg = tid / CG;
    const int w = __builtin_amdgcn_readfirstlane(tid / 64), lane = tid % 64;
    const int cb = (a.dv + CB - 1) / CB;
    const uint32_t item = xcd_item(blockIdx.x, (uint32_t)cb);
    if (item >= n_items) return;
    const int64_t bh = item / cb;
    const int64_t b = bh / a.Hv;
    const int h = (int)(bh - b * a.Hv), hk = h / a.rep;
    const int col = (int)(item - bh * cb) * CB + 4 * cg;
    const bool on = col < a.dv;
    int64_t slot = slots ? slots[b] : b;
    if (slots) {
        // the first entry that names a state has it
        if (tid == 0) sDup = 0;
        __syncthreads();
        bool dup = false;
        for (int64_t i = tid; i < b; i += 256) dup |= slots[i] == slot;
        if (dup) sDup = 1;
        __syncthreads();
        if (sDup) slot = -1;
    }
    if (slot < 0 || slot >= n_pool) {              // padding
        for (int64_t t = kg; t < L; t += KG)
            if (on) *(Raw4<T> *)(a.o.at<T>(b, h, t) + col) = zero4<T>();
        return;
    }
    float *st = pool + (slot * a.Hv + h) * a.dk * a.dv + col;
    floatx4 S[KPT];
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
        const int key = kg + KG * i;
        S[i] = on && key < a.dk ? *(const floatx4 *)(st + (int64_t)key * a.dv) : floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    for (int64_t t = 0; t < L; ++t) {
        float kq = 0.0f;
        if (tid < DK) {
            const float kx = tid < a.dk ? (float)a.k.at<const T>(b, hk, t)[tid] : 0.0f;
            const float qx = tid < a.dk ? (float)a.q.at<const T>(b, hk, t)[tid] : 0.0f;
            sKQ[0][tid] = kx;
            sKQ[1][tid] = qx;
            kq = kx * qx;
        }
#pragma unroll
        for (int m = 1; m < 64; m *= 2) kq += __shfl_xor(kq, m, 64);
        if (lane == 0) sDot[w] = kq;
        Raw4<T> v = zero4<T>();
        if (on) v = load4(a.v.at<const T>(b, h, t) + col);
        const float eg = expf(*a.g.at<const float>(b, h, t)), be = *a.beta.at<const float>(b, h, t);
        __syncthreads();
        floatx4 sk = {0.0f, 0.0f, 0.0f, 0.0f}, sq = sk;
#pragma unroll
        for (int i = 0; i < KPT; ++i) {
            const float kx = sKQ[0][kg + KG * i], qx = sKQ[1][kg + KG * i];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                S[i][j] *= eg;
                sk[j] = fmaf(S[i][j], kx, sk[j]);
                sq[j] = fmaf(S[i][j], qx, sq[j]);
            }
        }
#pragma unroll
        for (int m = CG; m < 64; m *= 2)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                sk[j] += __shfl_xor(sk[j], m, 64);
                sq[j] += __shfl_xor(sq[j], m, 64);
            }
        if (lane < CG) {
            sRed[w][0][lane] = sk;
            sRed[w][1][lane] = sq;
        }
        __syncthreads();
        sk = sRed[0][0][cg];
        sq = sRed[0][1][cg];
        float dot = sDot[0];
#pragma unroll
        for (int i = 1; i < 4; ++i) {
            const floatx4 x = sRed[i][0][cg], y = sRed[i][1][cg];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                sk[j] += x[j];
                sq[j] += y[j];
            }
            dot += sDot[i];
        }
        const floatx4 vf = v.f();
        float u[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) u[j] = be * (vf[j] - sk[j]);
#pragma unroll
        for (int i = 0; i < KPT; ++i) {
            const float kx = sKQ[0][kg + KG * i];
#pragma unroll
            for (int j = 0; j < 4; ++j) S[i][j] = fmaf(kx, u[j], S[i][j]);
        }
        if (on && kg == 0) {
            Raw4<T> o;
#pragma unroll
            for (int j = 0; j < 4; ++j) o.x[j] = (T)(a.scale * fmaf(dot, u[j], sq[j]));
            *(Raw4<T> *)(a.o.at<T>(b, h, t) + col) = o;
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
        const int key = kg + KG * i;
        if (on && key < a.dk) *(floatx4 *)(st + (int64_t)key * a.dv) = S[i];
    }
}

// ---------------------------------------------------------------- dispatch
static_assert(rec_bytes(true) == 3 * kMatBytes + 256 && rec_bytes(false) == 2 * kMatBytes + 256, "the planner's records");
View view(const void *p, const int64_t (&s)[3], int64_t H, int64_t L, int64_t d) {
    int64_t o[3];
    dense_strides(s, H, L, d, o);
    return View{p, o[0], o[1], o[2]};
}

Args make_args(const Plan &pl, const pgf_gdr_params *p, const void *q, const void *k, const void *v, const float *g,
               const float *beta, const void *o) {
    Args a{};
    a.q = view(q, p->q_strides, pl.Hk, pl.L, pl.dk);
    a.k = view(k, p->k_strides, pl.Hk, pl.L, pl.dk);
    a.v = view(v, p->v_strides, pl.Hv, pl.L, pl.dv);
    a.g = view(g, p->g_strides, pl.Hv, pl.L, 1);
    a.beta = view(beta, p->beta_strides, pl.Hv, pl.L, 1);
    a.o = view(o, p->o_strides, pl.Hv, pl.L, pl.dv);
    a.seqs = Seqs{p->n_seqs ? p->cu_seqlens : nullptr, pl.nseq, pl.L};
    a.chunk_per = pl.chunks_per;
    a.seg_per = pl.segs_per;
    a.seg = pl.seg;
    a.Hk = (int)pl.Hk;
    a.Hv = (int)pl.Hv;
    a.rep = (int)(pl.Hv / pl.Hk);
    a.dk = (int)pl.dk;
    a.dv = (int)pl.dv;
    a.scale = p->scale;
    a.vt = (int)((pl.dv + 15) / 16);
    a.ct = a.vt;
    return a;
}

// Pointers and overlaps of the arrays that every entry point has.
int check_arrays(const Plan &pl, const pgf_gdr_params *p, const void *q, const void *k, const void *v, const float *g,
                 const float *beta, const void *o) {
    if (p->n_seqs && !p->cu_seqlens) return PGF_ERR_INVALID_ARG;
    if (((uintptr_t)p->cu_seqlens | (uintptr_t)p->slots | (uintptr_t)p->S_in | (uintptr_t)p->S_out | (uintptr_t)p->dS_out |
         (uintptr_t)p->dS_in) & 3)
        return PGF_ERR_INVALID_ARG;
    if (pl.L == 0) return PGF_OK;
    if (!q || !k || !v || !g || !beta || !o) return PGF_ERR_INVALID_ARG;
    if (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)o) & 15) return PGF_ERR_INVALID_ARG;
    if (((uintptr_t)g | (uintptr_t)beta) & 3) return PGF_ERR_INVALID_ARG;
    return PGF_OK;
}

template <typename T, int DK>
int scan_t(Args a, const Plan &pl, const pgf_gdr_params *p, hipStream_t st) {
    {
        const int64_t items = pl.chunk_slots * pl.Hk;
        if (items) {
            Timed tm(0, st);
            hipLaunchKernelGGL((k_gdr_prep<T, DK>), dim3((unsigned)((items + kPrepWaves - 1) / kPrepWaves)),
                               dim3(64 * kPrepWaves), 0, st, a, pl.chunk_slots);
        }
    }
    a.S_in = p->S_in;
    a.S_out = p->S_out;
    if (pl.seg) {
        {
            Args s = a;
            s.ct = a.vt + (int)((pl.dk + 15) / 16);
            const uint32_t items = (uint32_t)(pl.seg_slots * pl.Hv * ((s.ct + 3) / 4));
            Timed tm(1, st);
            hipLaunchKernelGGL((k_gdr_chain<T, DK, kSegment, 1>), dim3((unsigned)xcd_grid(items, (s.ct + 3) / 4 * a.rep)), dim3(256), 0, st, s, items);
        }
        Timed tm(2, st);
        hipLaunchKernelGGL((k_gdr_carry<DK, false>), dim3((unsigned)xcd_grid(pl.nseq * pl.Hv * a.vt, a.vt)), dim3(4 * DK), 0, st, a);
        a.seg_in = a.segE;
    }
    Timed tm(3, st);
    const int cb = (a.ct * pl.share + 3) / 4;
    const uint32_t items = (uint32_t)(pl.seg_slots * pl.Hv * cb);
    const dim3 grid((unsigned)xcd_grid(items, cb * a.rep));
    if (pl.share == 2) hipLaunchKernelGGL((k_gdr_chain<T, DK, kOut, 2>), grid, dim3(256), 0, st, a, items);
    else hipLaunchKernelGGL((k_gdr_chain<T, DK, kOut, 1>), grid, dim3(256), 0, st, a, items);
    return hipGetLastError() == hipSuccess ? PGF_OK : PGF_ERR_HIP;
}

template <typename T>
int step_t(const Args &a, const Plan &pl, const pgf_gdr_params *p, hipStream_t st) {
    Timed tm(3, st);
    const int64_t cb = (pl.dv + pl.step_cols - 1) / pl.step_cols, items = pl.B * pl.Hv * cb;
    const dim3 grid((unsigned)xcd_grid(items, cb));
#define PGF_STEP(DK_, CB_) \
    hipLaunchKernelGGL((k_gdr_step<T, DK_, CB_>), grid, dim3(256), 0, st, a, p->S_pool, p->pool, p->slots, pl.L, (uint32_t)items)
    if (pl.DK == 64) {
        if (pl.step_cols == 128) PGF_STEP(64, 128); else PGF_STEP(64, 32);
    } else {
        if (pl.step_cols == 128) PGF_STEP(128, 128); else PGF_STEP(128, 32);
    }
#undef PGF_STEP
    return hipGetLastError() == hipSuccess ? PGF_OK : PGF_ERR_HIP;
}

}  // namespace gdr
}  // namespace pgf

extern "C" int pgf_gdr_scan(const void *q, const void *k, const void *v, const float *g, const float *beta,
                            const pgf_gdr_params *p, void *o, void *stream) {
    using namespace pgf;
    using namespace pgf::gdr;
    Plan pl;
    int rc = make_plan(p, &pl, false, false);
    if (rc != PGF_OK) return rc;
    rc = check_arrays(pl, p, q, k, v, g, beta, o);
    if (rc != PGF_OK) return rc;
    if (!p->workspace || p->workspace_bytes < pl.total || ((uintptr_t)p->workspace & 255)) return PGF_ERR_WORKSPACE;
    const size_t e = p->in_dtype == PGF_BF16 ? 2 : 4;
    const Arr out{o, p->o_strides, pl.B, pl.Hv, pl.L, pl.dv, e};
    const size_t ns = (size_t)(pl.nseq * pl.Hv * pl.dk * pl.dv) * 4;
    const int64_t dense[3] = {0, 0, 0};
    const Arr ins[] = {{q, p->q_strides, pl.B, pl.Hk, pl.L, pl.dk, e}, {k, p->k_strides, pl.B, pl.Hk, pl.L, pl.dk, e},
                       {v, p->v_strides, pl.B, pl.Hv, pl.L, pl.dv, e}, {g, p->g_strides, pl.B, pl.Hv, pl.L, 1, 4},
                       {beta, p->beta_strides, pl.B, pl.Hv, pl.L, 1, 4},
                       {p->n_seqs ? p->cu_seqlens : nullptr, dense, 1, 1, 1, pl.nseq + 1, 4}};
    for (const auto &i : ins)
        if (overlaps(out, i) || overlaps(p->workspace, pl.total, i.p, i.bytes()) || overlaps(p->S_out, ns, i.p, i.bytes()))
            return PGF_ERR_INVALID_ARG;
    // S_out may be S_in: a state is read before its sequence's last step writes it.
    if (overlaps(p->S_out, ns, p->S_in, ns) && p->S_out != p->S_in) return PGF_ERR_INVALID_ARG;
    const size_t no = out.bytes();
    if (overlaps(o, no, p->S_in, ns) || overlaps(o, no, p->S_out, ns) || overlaps(p->workspace, pl.total, o, no) ||
        overlaps(p->workspace, pl.total, p->S_in, ns) || overlaps(p->workspace, pl.total, p->S_out, ns))
        return PGF_ERR_INVALID_ARG;
    (void)hipGetLastError();
    Args a = make_args(pl, p, q, k, v, g, beta, o);
    char *ws = (char *)p->workspace;
    a.rec = ws + pl.rec;
    a.segE = (float *)(ws + pl.segE);
    a.tr = (float *)(ws + pl.tr);
    hipStream_t st = (hipStream_t)stream;
    const bool bf = p->in_dtype == PGF_BF16;
    if (p->clear_rest) {
        Rest rest{};
        rest.add(a.o, a.Hv, a.dv * (int)e, (int)e);
        clear_rest(rest, a, st);
    }
    if (pl.DK == 64) return bf ? scan_t<__bf16, 64>(a, pl, p, st) : scan_t<float, 64>(a, pl, p, st);
    return bf ? scan_t<__bf16, 128>(a, pl, p, st) : scan_t<float, 128>(a, pl, p, st);
}

extern "C" int pgf_gdr_step(const void *q, const void *k, const void *v, const float *g, const float *beta,
                            const pgf_gdr_params *p, void *o, void *stream) {
    using namespace pgf;
    using namespace pgf::gdr;
    Plan pl;
    int rc = make_plan(p, &pl, false, true);
    if (rc != PGF_OK) return rc;
    rc = check_arrays(pl, p, q, k, v, g, beta, o);
    if (rc != PGF_OK) return rc;
    if (!p->slots && p->pool < pl.B) return PGF_ERR_INVALID_ARG;
    if (p->pool && (!p->S_pool || ((uintptr_t)p->S_pool & 15))) return PGF_ERR_INVALID_ARG;
    const size_t e = p->in_dtype == PGF_BF16 ? 2 : 4;
    if ((double)p->pool * (double)(pl.Hv * pl.dk * pl.dv) > 1e18) return PGF_ERR_UNSUPPORTED;
    const Arr out{o, p->o_strides, pl.B, pl.Hv, pl.L, pl.dv, e};
    const size_t ns = (size_t)(p->pool * pl.Hv * pl.dk * pl.dv) * 4;
    const Arr ins[] = {{q, p->q_strides, pl.B, pl.Hk, pl.L, pl.dk, e}, {k, p->k_strides, pl.B, pl.Hk, pl.L, pl.dk, e},
                       {v, p->v_strides, pl.B, pl.Hv, pl.L, pl.dv, e}, {g, p->g_strides, pl.B, pl.Hv, pl.L, 1, 4},
                       {beta, p->beta_strides, pl.B, pl.Hv, pl.L, 1, 4}};
    for (const auto &i : ins)
        if (overlaps(out, i) || overlaps(p->S_pool, ns, i.p, i.bytes())) return PGF_ERR_INVALID_ARG;
    const size_t no = out.bytes(), nsl = (size_t)pl.B * 4;
    if (overlaps(o, no, p->S_pool, ns) || overlaps(o, no, p->slots, nsl) || overlaps(p->S_pool, ns, p->slots, nsl))
        return PGF_ERR_INVALID_ARG;
    if (pl.L == 0) return PGF_OK;
    (void)hipGetLastError();
    const Args a = make_args(pl, p, q, k, v, g, beta, o);
    return p->in_dtype == PGF_BF16 ? step_t<__bf16>(a, pl, p, (hipStream_t)stream)
                                   : step_t<float>(a, pl, p, (hipStream_t)stream);
}
