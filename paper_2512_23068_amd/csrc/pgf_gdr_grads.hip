// libpgf: gradients of the gated delta rule for gfx950.
//
// In the chunk form of pgf_gdr.hip, with E the errors (the steps write
// diag(beta) E), S0 and S1 the state entering and leaving a run of steps and
// dO, dS1 the adjoints of its outputs and of S1:
//   dE  = TW^T (K dS1) + scale TA^T dO                (dE is also dl/dV)
//   dS0 = e^{G_C} dS1 + Q^T (scale e^G dO) - K^T (e^G dE)
// so the adjoint runs through the chunks backwards with the forward chain's
// products transposed, and needs neither S nor E.  Everything else follows, for
// any run of steps (here 64), from E, dE, S0 and dS1.  With z_t = dS1 E_t,
// y_t = S0 dE_t, decays c_st = e^{G_s - G_t}, and sums over steps of the run:
//   dq_s = scale e^{G_s} S0 dO_s + sum_{t<=s} scale c_st beta_t (dO_s.E_t) k_t
//   w_t  = e^{G_C - G_t} z_t + sum_{s>=t} scale c_st (dO_s.E_t) q_s - sum_{s>t} c_st (dE_s.E_t) k_s
//   r_t  = -e^{G_t} y_t - sum_{u<t} c_tu beta_u (dE_t.E_u) k_u
//   dk_t = beta_t w_t + r_t,   dbeta_t = k_t.w_t
// dg_t is the sum of all that a step before t leaves to one from t on (each with the
// decays between, g_t among them): what q_s and k_s read less what k_u, u >= t, wrote
// of it, and what the steps before t and S0 leave to S1:
//   dg_t = sum_{s>=t} (q_s.dq'_s + k_s.r_s - beta_s k_s.w'_s) + sum_{u<t} e^{G_C - G_u} beta_u k_u.z_u
//          + e^{G_C} <dS1, S0>
// Here dq' is dq without its term t = s, and w' is w without its terms s = t and z:
// those have no decay and would cancel, and under strong decays dg is the small rest.
//
//   k_gdr_prep                records, with T^
//   k_gdr_chain<kSave>        forward: E, and S every 64 steps
//   k_gdr_back                backwards: dE, dl/dv, and dS every 64 steps
//   k_gdr_outer               per 64 steps and key head: dq, dk, dbeta, dg; the
//                             value heads of a key head one after the other, so
//                             their sums have an order
#include "pgf_gdr_chain.h"
#include "pgf_timing.h"

namespace pgf {
namespace gdr {

// ---------------------------------------------------------------- backwards
// As k_gdr_chain: a wave owns 16 value columns of the adjoint state of one head.
// kBackSegment: from zero at the segment's end to its start, nothing written on
// the way.
// Bound by issue like it: 2 x 4096 steps of 16 heads, 128 x 128 in bf16, 85 us and
// 64 us for kBackSegment (512 steps a segment; the forward chain 70 and 87 us).
template <typename T, int DK, int MODE>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void k_gdr_back(Args a, uint32_t n_items) {
    using Ck = Chunk<T, DK, MODE>;
    constexpr int P = Ck::P, NI = 6;
    constexpr int KS = DK / 32, KT = DK / 16;
    constexpr int KU = 32 * DK / 8 / 256, MU = 2;         // units of K, tiles of TW and TA a thread stages
    constexpr int NB = sizeof(Ck) <= 40960 ? 2 : 1;
    __shared__ Ck lds[NB];
    const int tid = threadIdx.x, lane = tid % 64, c = lane % 16, qd = lane / 16;
    const int w = __builtin_amdgcn_readfirstlane(tid / 64);
    const int cb = (a.vt + 3) / 4;
    const uint32_t item = xcd_item(blockIdx.x, (uint32_t)(cb * a.rep));
    if (item >= n_items) return;
    const int64_t sh = item / cb;
    const int tile = (int)(item - sh * cb) * 4 + w;
    const int64_t slot = sh / a.Hv;
    const int h = (int)(sh - slot * a.Hv), hk = h / a.rep;
    const Rows r = a.seqs.of(slot, a.seg ? a.seg : a.seqs.L + 1, a.seg_per);
    if (r.unit0 > 0 && r.unit0 >= r.len) return;   // uniform over the block
    if (MODE == kBackSegment && r.unit0 == 0) return;      // (nothing precedes it)
    int64_t n = uni(r.len - r.unit0);
    if (a.seg && n > a.seg) n = a.seg;
    const bool mine = tile < a.vt;
    const int col = tile * 16 + c;
    const bool live_col = mine && col < a.dv;
    const int chunks = (int)((n + kC - 1) / kC);
    const int64_t t0 = r.lo + r.unit0;
    const int64_t slot0 = uni(a.seqs.slot0(r.n, kC, a.chunk_per) + r.unit0 / kC);
    const int64_t save0 = uni(a.seqs.slot0(r.n, kC * kSuper, a.save_per) + r.unit0 / (kC * kSuper));

    floatx4 S[KT];                                 // the adjoint: key 32 (kt / 2) + 8 qd + 4 (kt % 2) + j
    const uint32_t est = (uint32_t)a.dv * 4, so = live_col ? (uint32_t)(8 * qd * a.dv + col) * 4u : kNone;
    const uint32_t eo = live_col ? (uint32_t)(4 * qd * a.dv + col) * 4u : kNone;
    auto state = [&](const float *p) {
        return Buf{__builtin_amdgcn_make_buffer_rsrc((void *)uni((int64_t)(uintptr_t)p), 0, a.dk * a.dv * 4, 0x00020000), est};
    };
    auto place = [&](int kt, int j) { return (uint32_t)(32 * (kt / 2) + 4 * (kt & 1) + j) * est; };
    {
        const float *in = MODE == kBackSegment ? nullptr : a.dseg_in && r.len ? a.dseg_in + (slot * a.Hv + h) * a.dk * a.dv
                          : a.dS_out ? a.dS_out + (r.n * a.Hv + h) * a.dk * a.dv : nullptr;
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) S[kt] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
        if (in) {
            const Buf ib = state(in);
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                for (int j = 0; j < 4; ++j) S[kt][j] = raw_f<float>(load1<float>(ib, so, place(kt, j)));
        }
    }
    auto store_state = [&](float *out) {
        const Buf ob = state(out);
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int j = 0; j < 4; ++j) store1<float>(ob, so, place(kt, j), S[kt][j]);
    };

    Raw8<T> rk[KU], rq[KU];
    uintx4 rm[MU];
    float reG;
    uint32_t ro[2][4];
    const T *kp = row_ptr<T>(a.k, r.b, hk, t0), *qp = row_ptr<T>(a.q, r.b, hk, t0), *gp = row_ptr<T>(a.go, r.b, h, t0),
            *vp = row_ptr<T>(a.dv_, r.b, h, t0);
    const uint32_t gst = (uint32_t)a.go.st * sizeof(T), vst = (uint32_t)a.dv_.st * sizeof(T);
    const uint32_t kst = (uint32_t)a.k.st * sizeof(T), qst = (uint32_t)a.q.st * sizeof(T);
    const uint32_t go = live_col ? 4 * qd * gst + col * (uint32_t)sizeof(T) : kNone;
    const uint32_t vo = live_col ? 4 * qd * vst + col * (uint32_t)sizeof(T) : kNone;
    const uint32_t rb = rec_bytes(true);
    uint32_t ko[KU], qo[KU];
#pragma unroll
    for (int i = 0; i < KU; ++i) {
        const int u = tid + 256 * i, t = u / (DK / 8), e = u % (DK / 8) * 8;
        ko[i] = e < a.dk ? t * kst + e * (uint32_t)sizeof(T) : kNone;
        qo[i] = e < a.dk ? t * qst + e * (uint32_t)sizeof(T) : kNone;
    }
    auto live_rows = [&](int ch) {
        const int64_t left = n - (int64_t)ch * kC;
        return (int)(left < kC ? left : kC);
    };
    auto fetch = [&](int ch) {
        const int live = live_rows(ch);
        const Buf kb = make_buf(kp + (int64_t)ch * kC * a.k.st, kst, live, a.dk * (int)sizeof(T));
        const Buf qb = make_buf(qp + (int64_t)ch * kC * a.q.st, qst, live, a.dk * (int)sizeof(T));
        const Buf gb = make_buf(gp + (int64_t)ch * kC * a.go.st, gst, live, a.dv * (int)sizeof(T));
#pragma unroll
        for (int i = 0; i < KU; ++i) {
            rk[i] = load8<T>(kb, ko[i], 0);
            rq[i] = load8<T>(qb, qo[i], 0);
        }
        const char *rec = a.rec + ((slot0 + ch) * a.Hv + h) * (int64_t)rb;
#pragma unroll
        for (int i = 0; i < MU; ++i) rm[i] = *(const uintx4 *)(rec + (w + 4 * i < 6 ? w + 4 * i : 0) * kTile + 16u * lane);
        reG = *(const float *)(rec + rec_eG(true) + 4 * (tid % 32));
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int j = 0; j < 4; ++j) ro[m][j] = load1<T>(gb, go, (16 * m + j) * gst);
    };
    auto stage = [&](Ck &s) {
#pragma unroll
        for (int i = 0; i < KU; ++i) {
            const int u = tid + 256 * i, t = u / (DK / 8);
            const uint32_t at = unit_off<DK>(t, u % (DK / 8));
            const Frag<P> f = raw_frag<P>(rk[i]), y = raw_frag<P>(rq[i]);
#pragma unroll
            for (int p = 0; p < P; ++p) {
                *(bf16x8 *)&s.K[p][at] = f.p[p];
                *(bf16x8 *)&s.Q[p][at] = y.p[p];
            }
        }
#pragma unroll
        for (int i = 0; i < MU; ++i) {
            const int t = w + 4 * i;
            if (t < 6) put_tile<3>(s.M + (t < 3 ? 0 : 3), t < 3 ? t : t - 3, rm[i]);
        }
        if (tid < 32) s.eG[tid] = reG;
    };

    if (chunks > 0) {
        fetch(chunks - 1);
        // dO's rows behind the end are inside its buffer where its step stride is
        // below a row.  (With them zero, Q's, K's and V's there count for nothing.)
        const int live = live_rows(chunks - 1);
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int j = 0; j < 4; ++j) ro[m][j] = 16 * m + 4 * qd + j < live ? ro[m][j] : 0u;
#pragma unroll
        for (int i = 0; i < NB; ++i) zero_tile<NI, 256>(lds[i].M, tid);
        stage(lds[0]);
        lds_barrier();
    }
    for (int i = 0; i < chunks; ++i) {
        const int ch = chunks - 1 - i;
        if constexpr (MODE == kBack)
            if (mine && (i == 0 || ch % kSuper == kSuper - 1))
                store_state(a.saveD + ((save0 + ch / kSuper) * a.Hv + h) * a.dk * a.dv);
        float g[2][4];
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int j = 0; j < 4; ++j) g[m][j] = raw_f<T>(ro[m][j]);
        const Ck &s = lds[NB == 2 ? i & 1 : 0];
        fetch(ch > 0 ? ch - 1 : 0);                // (the first chunk again rather than a branch)
        if (mine) {
            floatx4 x[2];
#pragma unroll
            for (int m = 0; m < 2; ++m) x[m] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
            Frag<P> kf[2][2];
            auto read_k = [&](int ks) {
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int p = 0; p < P; ++p)
                        kf[ks & 1][m].p[p] = *(const bf16x8 *)&s.K[p][unit_off<DK>(16 * m + c, 4 * ks + qd)];
            };
            // rows 16 m + c of the transposed images (TW^T: 0, TA^T: 3)
            auto read_mt = [&](int first, Frag<3> (&f)[2]) {
                const int row = 4 * qd + c / 4;
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int p = 0; p < 3; ++p) {
                        const char *m0 = &s.M[first + p][unit_off<32>(row, c % 4) + 8 * m];
                        const char *m1 = &s.M[first + p][unit_off<32>(16 + row, c % 4) + 8 * m];
                        f[m].p[p] = __builtin_shufflevector(read_tr(m0), read_tr(m1), 0, 1, 2, 3, 4, 5, 6, 7);
                    }
            };
            Frag<3> af[2], tf[2];
            floatx4 eG[2], dE[2];
            read_k(0);
            read_mt(3, af);
            const Frag<P> gf = to_frag<P>(floatx4{g[0][0], g[0][1], g[0][2], g[0][3]},
                                          floatx4{g[1][0], g[1][1], g[1][2], g[1][3]});
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                if (ks + 1 < KS) read_k(ks + 1);
                else {
                    read_mt(0, tf);
#pragma unroll
                    for (int m = 0; m < 2; ++m) eG[m] = *(const floatx4 *)&s.eG[16 * m + 4 * qd];
                }
                __builtin_amdgcn_sched_barrier(0);
                if (ks == 0) {
                    dE[0] = dE[1] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
                    mfma_parts2<3, P>(af, gf, dE);
                }
                const Frag<3> sp = to_frag<3>(S[2 * ks], S[2 * ks + 1]);
                mfma_parts2<P, 3>(kf[ks & 1], sp, x);
                __builtin_amdgcn_sched_barrier(0);
            }
            const Frag<3> xp = to_frag<3>(x[0], x[1]);
            constexpr int GK = P == 1 ? 4 : 1;
            Frag<P> ktf[2][GK], qtf[2][GK];
            auto read_kt = [&](int gr) {
#pragma unroll
                for (int e = 0; e < GK; ++e) {
                    const int kt = gr * GK + e, row = 4 * qd + c / 4;
                    const uint32_t o0 = unit_off<DK>(row, 4 * (kt / 2) + c % 4) + 8 * (kt & 1);
                    const uint32_t o1 = unit_off<DK>(16 + row, 4 * (kt / 2) + c % 4) + 8 * (kt & 1);
#pragma unroll
                    for (int p = 0; p < P; ++p) {
                        ktf[gr & 1][e].p[p] =
                            __builtin_shufflevector(read_tr(&s.K[p][o0]), read_tr(&s.K[p][o1]), 0, 1, 2, 3, 4, 5, 6, 7);
                        qtf[gr & 1][e].p[p] =
                            __builtin_shufflevector(read_tr(&s.Q[p][o0]), read_tr(&s.Q[p][o1]), 0, 1, 2, 3, 4, 5, 6, 7);
                    }
                }
            };
            read_kt(0);
            const float end = s.eG[31];
            __builtin_amdgcn_sched_barrier(0);
            floatx4 gs[2], es[2];
#pragma unroll
            for (int m = 0; m < 2; ++m) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    dE[m][j] *= a.scale;
                    gs[m][j] = a.scale * eG[m][j] * g[m][j];
                }
            }
            mfma_parts2<3, 3>(tf, xp, dE);
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int j = 0; j < 4; ++j) es[m][j] = -eG[m][j] * dE[m][j];
            const Frag<3> gp3 = to_frag<3>(gs[0], gs[1]), ep3 = to_frag<3>(es[0], es[1]);
#pragma unroll
            for (int gr = 0; gr < KT / GK; ++gr) {
                if (gr + 1 < KT / GK) read_kt(gr + 1);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int e = 0; e < GK; ++e)
#pragma unroll
                    for (int j = 0; j < 4; ++j) S[gr * GK + e][j] *= end;
#pragma unroll
                for (int sum = 2; sum >= 0; --sum)
#pragma unroll
                    for (int p = 0; p < P; ++p)
                        if (sum - p >= 0) {
#pragma unroll
                            for (int e = 0; e < GK; ++e)
                                S[gr * GK + e] = mfma(qtf[gr & 1][e].p[p], gp3.p[sum - p], S[gr * GK + e]);
#pragma unroll
                            for (int e = 0; e < GK; ++e)
                                S[gr * GK + e] = mfma(ktf[gr & 1][e].p[p], ep3.p[sum - p], S[gr * GK + e]);
                        }
                __builtin_amdgcn_sched_barrier(0);
            }
            if constexpr (MODE == kBack) {
                float *eb = a.saveU + ((slot0 + ch) * a.Hv + h) * (int64_t)(kC * a.dv);
                const Buf vb = make_buf(vp + (int64_t)ch * kC * a.dv_.st, vst, live_rows(ch), a.dv * (int)sizeof(T));
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int j = 0; j < 4; ++j) store1<T>(vb, vo, (16 * m + j) * vst, dE[m][j]);
                const Buf sb{__builtin_amdgcn_make_buffer_rsrc((void *)uni((int64_t)(uintptr_t)eb), 0, kC * a.dv * 4, 0x00020000), est};
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int j = 0; j < 4; ++j) store1<float>(sb, eo, (16 * m + j) * est, dE[m][j]);
            }
        }
        if constexpr (NB == 1) lds_barrier();
        stage(lds[NB == 2 ? (i + 1) & 1 : 0]);
        lds_barrier();
    }
    if (!mine) return;
    if constexpr (MODE == kBackSegment) store_state(a.dsegE + (slot * a.Hv + h) * a.dk * a.dv);
    else if (a.dS_in && r.unit0 == 0) store_state(a.dS_in + (r.n * a.Hv + h) * a.dk * a.dv);
}

// ---------------------------------------------------------------- outer
// A block takes 64 steps of one key head; wave w of a side their tile of 16 steps
// 16 w .. as columns of every product, and all keys as rows, so that the sums over
// keys (dbeta, dG) stay in a wave.  Four waves are side 0, which has what reads the
// state (y, S0 dO and the products with earlier steps: dq, r), four side 1, which
// has what writes it (z and the products with later steps: w); a SIMD holds a wave
// of each.  Phase one runs over the value columns, 32 at a time through LDS in
// three parts, which both sides read: the products with S0 (or dS1), and the
// 64 x 64 products of E, dE and dO in the orientation the next product wants them
// as operand.  Phase two adds the products with K and Q, and r passes to side 1.
// At 128 x 128 in bf16 a block takes about 95000 cycles, 29000 of them in a SIMD's
// matrix instructions: the rest is the staging (7 instructions for two numbers'
// parts) and the waits between the phases, which one block of eight waves a CU (all
// that the registers hold) does not fill.  1024 blocks of two heads (2 x 4096
// steps, 16 heads) take 190 us; two blocks of four waves a CU, one side after the
// other with S0, E and dE read and split twice, took 220 us.
constexpr int kRun = kC * kSuper;
constexpr double kLog2e = 1.4426950408889634;

template <typename T, int DK>
struct OuterLds {
    static constexpr int P = sizeof(T) == 2 ? 1 : 3;
    struct Cols {
        __align__(16) char S[2][3][DK * 64];       // S0, dS1: rows of 32 value columns
        __align__(16) char E[2][3][kRun * 64], dO[P][kRun * 64];       // E and dE
    };
    // Two in LDS where they fit: one barrier per 32 columns.
    static constexpr int NB = 2 * sizeof(Cols) <= 155 * 1024 ? 2 : 1;
    union {
        Cols v[NB];
        struct {
            __align__(16) char K[P][kRun * DK * 2], Q[P][kRun * DK * 2];
            __align__(16) floatx4 r[4 * (DK / 16) * 64];               // [wave][kt][lane]
        } k;
    };
    double G[kRun];                                // sums of g, in powers of two
    float be[kRun], dG[2][kRun], kz[kRun], dot[8];
};

// One side of all value heads of a key head.  accq, acck: f32 sums on their way
// over the value heads, in the workspace: each place is written and read by one
// lane.  In registers they left too few for the products' operands.
template <typename T, int DK, int SIDE>
__device__ __forceinline__ void outer_side(const Args &a, OuterLds<T, DK> &lds, const Rows &r, int64_t t0, int live,
                                           int64_t slot0, int64_t sslot, int hk, int w, float *accq, float *acck) {
    using Lds = OuterLds<T, DK>;
    constexpr int P = Lds::P, NB = Lds::NB;
    constexpr int KT = DK / 16, KU = kRun * DK / 8 / 256;
    // Tiles of 16 rows at a time in the products: two, so that those that add to
    // the same tile wait less for each other, where their parts leave registers.
    constexpr int W = P == 1 ? 2 : 1;
    // The block's 128 rows of threads stage S0 and dS1, one row of each; where a
    // state has 64 rows side 0 stages S0 and side 1 dS1.
    constexpr bool S0 = DK == 128 || SIDE == 0, D1 = DK == 128 || SIDE == 1;
    const int lane = threadIdx.x % 64;
    int c = lane % 16, qd = lane / 16, tid = threadIdx.x;
    Raw8<float> r0, r1, re;                        // rows of S0 and dS1, of E (side 0) or dE (side 1)
    Raw8<T> rg;                                    // of dO (side 1)
    float gl, bl;                                  // g and beta of step `lane`
    auto fetch = [&](int vh, int v0) {
        const int h = hk * a.rep + vh, eu = tid % 4, er = tid % 256 / 4, sr = DK == 128 ? tid / 4 : er;
        const int64_t cell = (sslot * a.Hv + h) * (int64_t)(a.dk * a.dv);
        const Buf s0b = make_buf((const void *)uni((int64_t)(uintptr_t)(a.saveS + cell)), a.dv * 4, a.dk, a.dv * 4);
        const Buf s1b = make_buf((const void *)uni((int64_t)(uintptr_t)(a.saveD + cell)), a.dv * 4, a.dk, a.dv * 4);
        const bool con = v0 + 8 * eu < a.dv;       // this thread's columns are there
        const uint32_t vc = (uint32_t)(v0 + 8 * eu);
        const uint32_t at = con ? (uint32_t)sr * (a.dv * 4u) + vc * 4u : kNone;
        r0 = load8<float>(s0b, at, 0);             // (side 1 for <dS1, S0>)
        if constexpr (D1) r1 = load8<float>(s1b, at, 0);
        const int64_t row0 = ((slot0 + (er < live ? er / kC : 0)) * a.Hv + h) * (int64_t)(kC * a.dv) + (er < live ? er % kC * a.dv : 0);
        const float *ep = (SIDE ? a.saveU : a.saveE) + row0 + (con ? vc : 0);
        re.x = *(const uintx4 *)ep;
        re.y = *(const uintx4 *)(ep + 4);
        if constexpr (SIDE == 1) {
            const Buf gb = make_buf(row_ptr<T>(a.go, r.b, h, t0), (uint32_t)a.go.st * sizeof(T), live, a.dv * (int)sizeof(T));
            // (a step stride below a row leaves rows behind the end inside the buffer)
            rg = load8<T>(gb, con && er < live ? er * gb.st + vc * (uint32_t)sizeof(T) : kNone, 0);
        }
    };
    auto gates = [&](int vh) {
        const int64_t t = t0 + (lane < live ? lane : 0);
        gl = *a.g.at<const float>(r.b, hk * a.rep + vh, t);
        bl = *a.beta.at<const float>(r.b, hk * a.rep + vh, t);
    };
    float ss = 0.0f;                               // <dS1, S0>
    auto stage = [&](typename Lds::Cols &v, int v0) {
        const int eu = tid % 4, er = tid % 256 / 4, sr = DK == 128 ? tid / 4 : er;
        const uint32_t at = unit_off<32>(er, eu), sat = unit_off<32>(sr, eu);
        Raw8<float> me = re;
        if (!(v0 + 8 * eu < a.dv && er < live)) me.x = me.y = uintx4{};
        const Frag<3> fe = raw_frag<3>(me);
#pragma unroll
        for (int p = 0; p < 3; ++p) *(bf16x8 *)&v.E[SIDE][p][at] = fe.p[p];
        if constexpr (SIDE == 1) {
            const Frag<P> fg = raw_frag<P>(rg);
#pragma unroll
            for (int p = 0; p < P; ++p) *(bf16x8 *)&v.dO[p][at] = fg.p[p];
        }
        if constexpr (S0) {
            const Frag<3> f = raw_frag<3>(r0);
#pragma unroll
            for (int p = 0; p < 3; ++p) *(bf16x8 *)&v.S[0][p][sat] = f.p[p];
        }
        if constexpr (D1) {
            const Frag<3> f = raw_frag<3>(r1);
#pragma unroll
            for (int p = 0; p < 3; ++p) *(bf16x8 *)&v.S[1][p][sat] = f.p[p];
            const floatx4 a0 = __builtin_bit_cast(floatx4, r0.x), a1 = __builtin_bit_cast(floatx4, r1.x);
            const floatx4 b0 = __builtin_bit_cast(floatx4, r0.y), b1 = __builtin_bit_cast(floatx4, r1.y);
#pragma unroll
            for (int j = 0; j < 4; ++j) ss = fmaf(a0[j], a1[j], fmaf(b0[j], b1[j], ss));
        }
    };
    fetch(0, 0);
    gates(0);
    for (int vh = 0; vh < a.rep; ++vh) {
    const int h = hk * a.rep + vh;
    // The lane's place, hidden from the compiler's motion of what does not
    // change out of the loop: the LDS addresses of both phases, kept over the
    // loop, took a hundred registers more than there are.
    asm volatile("" : "+v"(c), "+v"(qd), "+v"(tid));
    // ---- phase one
    floatx4 x1[KT], x2[SIDE ? 1 : KT], d1[4], d2[4];      // side 0: y, S0 dO; side 1: z
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
        x1[kt] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
        if constexpr (SIDE == 0) x2[kt] = x1[kt];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) d1[i] = d2[i] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    ss = 0.0f;
    if (vh) lds_barrier();                         // the last head's reads
    stage(lds.v[0], 0);
    if (SIDE == 0 && w == 3) {
        double G = lane < live ? (gl < -200.0f ? -200.0f : gl) : 0.0f;
#pragma unroll
        for (int m = 1; m < 64; m *= 2) {
            const double o = __shfl_up(G, m, 64);
            if (lane >= m) G += o;
        }
        lds.G[lane] = G * kLog2e;
        lds.be[lane] = lane < live ? bl : 0.0f;
    }
    const int more = vh + 1 < a.rep ? vh + 1 : vh;
    fetch(a.dv > 32 ? vh : more, a.dv > 32 ? 32 : 0);
    lds_barrier();
    for (int v0 = 0; v0 < a.dv; v0 += 32) {
        const typename Lds::Cols &v = lds.v[NB == 2 ? v0 / 32 & 1 : 0];
        // (operands are read W tiles ahead, and no further: more take registers)
        const uint32_t wa = unit_off<32>(16 * w + c, qd);      // this wave's steps as columns
        Frag<3> f[2][W];
        auto read = [&](int n) {               // rows of S0 (dS1), then of E (dE)
#pragma unroll
            for (int i = 0; i < W; ++i)
#pragma unroll
                for (int p = 0; p < 3; ++p)
                    f[n & 1][i].p[p] = n < KT / W
                        ? *(const bf16x8 *)&v.S[SIDE][p][unit_off<32>(16 * (W * n + i) + c, qd)]
                        : *(const bf16x8 *)&v.E[SIDE][p][unit_off<32>(16 * (W * (n - KT / W) + i) + c, qd)];
        };
        Frag<3> xw;                            // dE or E
        Frag<P> gw;
#pragma unroll
        for (int p = 0; p < 3; ++p) xw.p[p] = *(const bf16x8 *)&v.E[1 - SIDE][p][wa];
        if constexpr (SIDE == 0) {
#pragma unroll
            for (int p = 0; p < P; ++p) gw.p[p] = *(const bf16x8 *)&v.dO[p][wa];
        }
        read(0);
#pragma unroll
        for (int n = 0; n < (KT + 4) / W; ++n) {
            if (n + 1 < (KT + 4) / W) read(n + 1);
            const int i = W * (n - KT / W);
            Frag<P> fg[W];
            if (SIDE == 1 && n >= KT / W) {
#pragma unroll
                for (int j = 0; j < W; ++j)
#pragma unroll
                    for (int p = 0; p < P; ++p) fg[j].p[p] = *(const bf16x8 *)&v.dO[p][unit_off<32>(16 * (i + j) + c, qd)];
            }
            __builtin_amdgcn_sched_barrier(0);
            const Frag<3> (&fp)[W] = f[n & 1];
            if (n < KT / W) {
                mfma_parts2<3, 3>(fp, xw, x1 + W * n);
                if constexpr (SIDE == 0) mfma_parts2<3, P>(fp, gw, x2 + W * n);
            } else {
                mfma_parts2<3, 3>(fp, xw, d2 + i);
                if constexpr (SIDE == 0) mfma_parts2<3, P>(fp, gw, d1 + i);
                else mfma_parts2<P, 3>(fg, xw, d1 + i);
            }
        }
        if (v0 + 32 >= a.dv) break;
        if constexpr (NB == 1) lds_barrier();
        stage(lds.v[NB == 2 ? (v0 / 32 + 1) & 1 : 0], v0 + 32);
        const bool on = v0 + 64 < a.dv;        // these columns of this head follow, or the next head's first
        fetch(on ? vh : more, on ? v0 + 64 : 0);
        lds_barrier();
    }
    gates(more);
    // ---- phase two
    asm volatile("" : "+v"(c), "+v"(qd), "+v"(tid));
    const int tok = 16 * w + c;                // this lane's step
    const View &kq = SIDE ? a.q : a.k;         // this side stages
    Raw8<T> rk[KU];
    {
        const Buf kb = make_buf(row_ptr<T>(kq, r.b, hk, t0), (uint32_t)kq.st * sizeof(T), live, a.dk * (int)sizeof(T));
#pragma unroll
        for (int i = 0; i < KU; ++i) {
            const int u = tid % 256 + 256 * i, t = u / (DK / 8), e = u % (DK / 8) * 8;
            rk[i] = load8<T>(kb, e < a.dk ? t * kb.st + e * (uint32_t)sizeof(T) : kNone, 0);
        }
    }
#pragma unroll
    for (int m = 1; m < 64; m *= 2) ss += __shfl_xor(ss, m, 64);
    if (lane == 0) lds.dot[4 * SIDE + w] = ss;
    const double Gt = lds.G[tok], Gend = lds.G[kRun - 1];
    const float be = lds.be[tok];
    // decays and signs of the 64 x 64 products; what has no place is zero.  The step's
    // own term, scale dO_t.E_t, stays apart.
    float own = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int row = 16 * i + 4 * qd + j;
            const float dG = (float)(Gt - lds.G[row]);
            const bool at = SIDE ? row > tok : row < tok;
            const float e = __builtin_amdgcn_exp2f(at ? (SIDE ? -dG : dG) : 0.0f) * (SIDE ? 1.0f : lds.be[row]);
            own = row == tok ? d1[i][j] : own;
            d1[i][j] = at ? a.scale * e * d1[i][j] : 0.0f;
            d2[i][j] = at ? -e * d2[i][j] : 0.0f;
        }
    own = a.scale * (SIDE ? 1.0f : be) * __shfl(own, c / 4 * 16 + c, 64);
    lds_barrier();                             // phase one's reads
#pragma unroll
    for (int i = 0; i < KU; ++i) {
        const int u = tid % 256 + 256 * i, t = u / (DK / 8);
        const uint32_t at = unit_off<DK>(t, u % (DK / 8));
        const Frag<P> f = raw_frag<P>(rk[i]);
#pragma unroll
        for (int p = 0; p < P; ++p) *(bf16x8 *)&(SIDE ? lds.k.Q : lds.k.K)[p][at] = f.p[p];
    }
    lds_barrier();
    // this lane's place in the sums over heads (what is not there, or not yet
    // written, is some place of them: loads without conditions)
    auto acc_at = [&](const float *acc, int kt) {
        const int key = 16 * kt + 4 * qd;
        return (const floatx4 *)(acc + (vh && key < a.dk ? tok * a.dk + key : 0));
    };
    // the sums go on to the next head, or out
    auto keep = [&](const View &o, float *acc, const floatx4 (&x)[KT]) {
        if (vh + 1 < a.rep) {
            const Buf b{__builtin_amdgcn_make_buffer_rsrc((void *)uni((int64_t)(uintptr_t)acc), 0, kRun * a.dk * 4, 0x00020000), 0};
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) {
                const uint32_t key = 16 * kt + 4 * qd;
                __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(uintx4, x[kt]), b.r,
                                                       (int)key < a.dk ? (tok * a.dk + key) * 4u : kNone, 0, 0);
            }
            return;
        }
        const Buf b = make_buf(row_ptr<T>(o, r.b, hk, t0), (uint32_t)o.st * sizeof(T), live, a.dk * (int)sizeof(T));
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
            const uint32_t key = 16 * kt + 4 * qd, at = (int)key < a.dk && tok < live ? tok * b.st + key * (uint32_t)sizeof(T) : kNone;
            if constexpr (sizeof(T) == 4) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(uintx4, x[kt]), b.r, at, 0, 0);
            else __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(uintx2, __builtin_convertvector(x[kt], bf16x4)), b.r, at, 0, 0);
        }
    };
    // keys 16 kt + 4 qd .. of this lane's step
    auto row4 = [&](const char (*m)[kRun * DK * 2], int kt) {
        floatx4 x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int p = P - 1; p >= 0; --p)
            x += __builtin_convertvector(*(const bf16x4 *)&m[p][unit_off<DK>(tok, 2 * kt + qd / 2) + 8 * (qd & 1)], floatx4);
        return x;
    };
    // operand of keys 16 kt .. and the 32 steps of block b, transposed
    auto tr = [&](const char (*m)[kRun * DK * 2], int b, int kt) {
        Frag<P> f;
        const int row = 32 * b + 4 * qd + c / 4, p4 = c % 4;
        const uint32_t o0 = unit_off<DK>(row, 2 * kt + p4 / 2) + 8 * (p4 & 1);
        const uint32_t o1 = unit_off<DK>(row + 16, 2 * kt + p4 / 2) + 8 * (p4 & 1);
#pragma unroll
        for (int p = 0; p < P; ++p)
            f.p[p] = __builtin_shufflevector(read_tr(&m[p][o0]), read_tr(&m[p][o1]), 0, 1, 2, 3, 4, 5, 6, 7);
        return f;
    };
    if constexpr (SIDE == 0) {
        const float eG = __builtin_amdgcn_exp2f((float)Gt);
        float qdq = 0.0f, kr = 0.0f;
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x1[kt][j] *= -eG;
                x2[kt][j] *= a.scale * eG;
            }
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            if (2 * b > w) continue;           // (uniform over the wave)
            const Frag<3> f1 = to_frag<3>(d1[2 * b], d1[2 * b + 1]), f2 = to_frag<3>(d2[2 * b], d2[2 * b + 1]);
            Frag<P> kf[2][W];
            auto read = [&](int kt) {
#pragma unroll
                for (int i = 0; i < W; ++i) kf[kt / W & 1][i] = tr(lds.k.K, b, kt + i);
            };
            read(0);
#pragma unroll
            for (int kt = 0; kt < KT; kt += W) {
                const int x = kt / W & 1;
                if (kt + W < KT) read(kt + W);
                __builtin_amdgcn_sched_barrier(0);
                mfma_parts2<P, 3>(kf[x], f1, x2 + kt);
                mfma_parts2<P, 3>(kf[x], f2, x1 + kt);
            }
        }
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
            const floatx4 kx = row4(lds.k.K, kt), qx = row4(lds.k.Q, kt);
            if (kt % 2 == 0) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                kr = fmaf(kx[j], x1[kt][j], kr);
                qdq = fmaf(qx[j], x2[kt][j], qdq);
                x2[kt][j] = fmaf(own, kx[j], x2[kt][j]);
            }
        }
        float s = qdq + kr;
#pragma unroll
        for (int m = 16; m < 64; m *= 2) s += __shfl_xor(s, m, 64);
        if (qd == 0) lds.dG[0][tok] = s;
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) lds.k.r[(w * KT + kt) * 64 + lane] = x1[kt];
        floatx4 sum[KT];                       // of the heads before
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) sum[kt] = *acc_at(accq, kt);
        lds_barrier();
        if (vh) {
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) x2[kt] += sum[kt];
        }
        keep(a.dq, accq, x2);
    } else {
        const float out = __builtin_amdgcn_exp2f((float)(Gend - Gt));
        float kz = 0.0f, kw = 0.0f, kq = 0.0f;         // k.z, k.w', k.q
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
            const floatx4 kx = row4(lds.k.K, kt);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x1[kt][j] *= out;
                kz = fmaf(kx[j], x1[kt][j], kz);
            }
        }
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            if (2 * b + 1 < w) continue;
            const Frag<3> f1 = to_frag<3>(d1[2 * b], d1[2 * b + 1]), f2 = to_frag<3>(d2[2 * b], d2[2 * b + 1]);
            Frag<P> qf[2][W], kf[2][W];
            auto read = [&](int kt) {
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    qf[kt / W & 1][i] = tr(lds.k.Q, b, kt + i);
                    kf[kt / W & 1][i] = tr(lds.k.K, b, kt + i);
                }
            };
            read(0);
#pragma unroll
            for (int kt = 0; kt < KT; kt += W) {
                const int x = kt / W & 1;
                if (kt + W < KT) read(kt + W);
                __builtin_amdgcn_sched_barrier(0);
                floatx4 y[W], v[W];
#pragma unroll
                for (int i = 0; i < W; ++i) y[i] = v[i] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
                mfma_parts2<P, 3>(qf[x], f1, v);
                mfma_parts2<P, 3>(kf[x], f2, y);
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    const floatx4 kx = row4(lds.k.K, kt + i), s = y[i] + v[i];
#pragma unroll
                    for (int j = 0; j < 4; ++j) kw = fmaf(kx[j], s[j], kw);
                    x1[kt + i] += s;
                }
            }
        }
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
            const floatx4 kx = row4(lds.k.K, kt), qx = row4(lds.k.Q, kt);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                kq = fmaf(kx[j], qx[j], kq);
                x1[kt][j] = fmaf(own, qx[j], x1[kt][j]);
            }
        }
#pragma unroll
        for (int m = 16; m < 64; m *= 2) {
            kz += __shfl_xor(kz, m, 64);
            kw += __shfl_xor(kw, m, 64);
            kq += __shfl_xor(kq, m, 64);
        }
        if (qd == 0) {
            lds.dG[1][tok] = -be * kw;
            lds.kz[tok] = be * kz;
            if (tok < live) a.dbeta[(r.b * a.Hv + h) * a.seqs.L + t0 + tok] = fmaf(own, kq, kz + kw);
        }
        floatx4 sum[KT];
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) sum[kt] = *acc_at(acck, kt);
        lds_barrier();
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
            const floatx4 rx = lds.k.r[(w * KT + kt) * 64 + lane];
#pragma unroll
            for (int j = 0; j < 4; ++j) x1[kt][j] = fmaf(be, x1[kt][j], rx[j]);
            if (vh) x1[kt] += sum[kt];
        }
        keep(a.dk_, acck, x1);
        if (w == vh % 4) {
            double v = (double)lds.dG[0][lane] + lds.dG[1][lane], e = lane ? lds.kz[lane - 1] : 0.0;
#pragma unroll
            for (int m = 1; m < 64; m *= 2) {
                const double x = __shfl_down(v, m, 64), y = __shfl_up(e, m, 64);
                if (lane + m < 64) v += x;
                if (lane >= m) e += y;
            }
            double s01 = 0.0;
#pragma unroll
            for (int i = 0; i < 8; ++i) s01 += lds.dot[i];
            if (lane < live)
                a.dg[(r.b * a.Hv + h) * a.seqs.L + t0 + lane] =
                    (float)(v + e + (double)__builtin_amdgcn_exp2f((float)lds.G[kRun - 1]) * s01);
        }
    }
    }
}

template <typename T, int DK>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2))) void k_gdr_outer(Args a) {
    __shared__ OuterLds<T, DK> lds;
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), w = wv % 4;
    const int64_t sslot = blockIdx.x / a.Hk;
    const int hk = (int)(blockIdx.x - sslot * a.Hk);
    const Rows r = a.seqs.of(sslot, kRun, a.save_per);
    if (r.unit0 >= r.len) return;                  // uniform over the block
    const int live = (int)uni(r.len - r.unit0 < kRun ? r.len - r.unit0 : kRun);
    const int64_t t0 = uni(r.lo + r.unit0);
    const int64_t slot0 = uni(a.seqs.slot0(r.n, kC, a.chunk_per) + r.unit0 / kC);

    // (with one value head a key head nothing is kept there, and its first bytes are read in vain)
    float *const accq = a.acc + (a.rep > 1 ? (sslot * a.Hk + hk) * (int64_t)(2 * kRun * a.dk) : 0);
    float *const acck = accq + (a.rep > 1 ? kRun * a.dk : 0);
    // (the sides pass the same number of barriers)
    if (wv < 4) outer_side<T, DK, 0>(a, lds, r, t0, live, slot0, sslot, hk, w, accq, acck);
    else outer_side<T, DK, 1>(a, lds, r, t0, live, slot0, sslot, hk, w, accq, acck);
}

// ---------------------------------------------------------------- dispatch
View view(const void *p, const int64_t (&s)[3], int64_t H, int64_t L, int64_t d);
Args make_args(const Plan &pl, const pgf_gdr_params *p, const void *q, const void *k, const void *v, const float *g,
               const float *beta, const void *o);
int check_arrays(const Plan &pl, const pgf_gdr_params *p, const void *q, const void *k, const void *v, const float *g,
                 const float *beta, const void *o);

template <typename T, int DK>
int grads_t(Args a, const Plan &pl, hipStream_t st) {
    const int64_t items = pl.chunk_slots * pl.Hk;
    if (items) {
        Timed tm(0, st);
        hipLaunchKernelGGL((k_gdr_prep<T, DK>), dim3((unsigned)((items + kPrepWaves - 1) / kPrepWaves)),
                           dim3(64 * kPrepWaves), 0, st, a, pl.chunk_slots);
    }
    if (pl.seg) {
        {
            Args s = a;
            s.ct = a.vt + (int)((pl.dk + 15) / 16);
            const uint32_t n = (uint32_t)(pl.seg_slots * pl.Hv * ((s.ct + 3) / 4));
            Timed tm(1, st);
            hipLaunchKernelGGL((k_gdr_chain<T, DK, kSegment, 1>), dim3((unsigned)xcd_grid(n, (s.ct + 3) / 4 * a.rep)), dim3(256), 0, st, s, n);
        }
        {
            const uint32_t n = (uint32_t)(pl.seg_slots * pl.Hv * ((a.vt + 3) / 4));
            Timed tm(1, st);
            hipLaunchKernelGGL((k_gdr_back<T, DK, kBackSegment>), dim3((unsigned)xcd_grid(n, (a.vt + 3) / 4 * a.rep)), dim3(256), 0, st, a, n);
        }
        Timed tm(2, st);
        hipLaunchKernelGGL((k_gdr_carry<DK, true>), dim3((unsigned)xcd_grid(pl.nseq * pl.Hv * a.vt, a.vt), 2), dim3(4 * DK), 0, st, a);
        a.seg_in = a.segE;
        a.dseg_in = a.dsegE;
    }
    const uint32_t blocks = (uint32_t)(pl.seg_slots * pl.Hv * ((a.ct + 3) / 4));
    if (items) {
        Timed tm(1, st);
        hipLaunchKernelGGL((k_gdr_chain<T, DK, kSave, 1>), dim3((unsigned)xcd_grid(blocks, (a.vt + 3) / 4 * a.rep)), dim3(256), 0, st, a, blocks);
    }
    {
        Timed tm(2, st);
        hipLaunchKernelGGL((k_gdr_back<T, DK, kBack>), dim3((unsigned)xcd_grid(blocks, (a.vt + 3) / 4 * a.rep)), dim3(256), 0, st, a, blocks);
    }
    if (items) {
        Timed tm(3, st);
        const uint32_t n = (uint32_t)(pl.super_slots * pl.Hk);
        hipLaunchKernelGGL((k_gdr_outer<T, DK>), dim3(n), dim3(512), 0, st, a);
    }
    return hipGetLastError() == hipSuccess ? PGF_OK : PGF_ERR_HIP;
}

}  // namespace gdr
}  // namespace pgf

extern "C" int pgf_gdr_grads(const void *q, const void *k, const void *v, const float *g, const float *beta,
                             const void *do_, const pgf_gdr_params *p, void *dq, void *dk, void *dv, float *dg,
                             float *dbeta, void *stream) {
    using namespace pgf;
    using namespace pgf::gdr;
    Plan pl;
    int rc = make_plan(p, &pl, true, false);
    if (rc != PGF_OK) return rc;
    rc = check_arrays(pl, p, q, k, v, g, beta, do_);
    if (rc != PGF_OK) return rc;
    if (pl.L > 0 && (!dq || !dk || !dv || !dg || !dbeta)) return PGF_ERR_INVALID_ARG;
    if (((uintptr_t)dq | (uintptr_t)dk | (uintptr_t)dv) & 15) return PGF_ERR_INVALID_ARG;
    if (((uintptr_t)dg | (uintptr_t)dbeta) & 3) return PGF_ERR_INVALID_ARG;
    if (!p->workspace || p->workspace_bytes < pl.total || ((uintptr_t)p->workspace & 255)) return PGF_ERR_WORKSPACE;
    const size_t e = p->in_dtype == PGF_BF16 ? 2 : 4;
    const size_t ns = (size_t)(pl.nseq * pl.Hv * pl.dk * pl.dv) * 4, ng = (size_t)(pl.B * pl.Hv * pl.L) * 4;
    const int64_t dense[3] = {0, 0, 0};
    const Arr ins[] = {{q, p->q_strides, pl.B, pl.Hk, pl.L, pl.dk, e}, {k, p->k_strides, pl.B, pl.Hk, pl.L, pl.dk, e},
                       {v, p->v_strides, pl.B, pl.Hv, pl.L, pl.dv, e}, {do_, p->o_strides, pl.B, pl.Hv, pl.L, pl.dv, e},
                       {g, p->g_strides, pl.B, pl.Hv, pl.L, 1, 4}, {beta, p->beta_strides, pl.B, pl.Hv, pl.L, 1, 4},
                       {p->S_in, dense, 1, 1, 1, (int64_t)ns, 1}, {p->dS_out, dense, 1, 1, 1, (int64_t)ns, 1},
                       {p->n_seqs ? p->cu_seqlens : nullptr, dense, 1, 1, 1, pl.nseq + 1, 4}};
    const Arr outs[] = {{dq, p->dq_strides, pl.B, pl.Hk, pl.L, pl.dk, e}, {dk, p->dk_strides, pl.B, pl.Hk, pl.L, pl.dk, e},
                        {dv, p->dv_strides, pl.B, pl.Hv, pl.L, pl.dv, e}, {dg, dense, 1, 1, 1, (int64_t)ng, 1},
                        {dbeta, dense, 1, 1, 1, (int64_t)ng, 1}, {p->dS_in, dense, 1, 1, 1, (int64_t)ns, 1}};
    const Arr ws_{p->workspace, dense, 1, 1, 1, (int64_t)pl.total, 1};
    for (int i = 0; i < 6; ++i) {
        for (const auto &x : ins)
            if (overlaps(outs[i], x)) return PGF_ERR_INVALID_ARG;
        for (int j = 0; j < i; ++j)
            if (overlaps(outs[i], outs[j])) return PGF_ERR_INVALID_ARG;
        if (overlaps(outs[i], ws_)) return PGF_ERR_INVALID_ARG;
    }
    for (const auto &x : ins)
        if (overlaps(x, ws_)) return PGF_ERR_INVALID_ARG;
    (void)hipGetLastError();
    Args a = make_args(pl, p, q, k, v, g, beta, nullptr);
    a.go = view(do_, p->o_strides, pl.Hv, pl.L, pl.dv);
    a.dq = view(dq, p->dq_strides, pl.Hk, pl.L, pl.dk);
    a.dk_ = view(dk, p->dk_strides, pl.Hk, pl.L, pl.dk);
    a.dv_ = view(dv, p->dv_strides, pl.Hv, pl.L, pl.dv);
    char *ws = (char *)p->workspace;
    a.rec = ws + pl.rec;
    a.grads = 1;
    a.segE = (float *)(ws + pl.segE);
    a.tr = (float *)(ws + pl.tr);
    a.trT = (float *)(ws + pl.trT);
    a.S_in = p->S_in;
    a.dS_out = p->dS_out;
    a.dS_in = p->dS_in;
    a.saveS = (float *)(ws + pl.S);
    a.saveD = (float *)(ws + pl.dS);
    a.saveE = (float *)(ws + pl.u);
    a.saveU = (float *)(ws + pl.du);
    a.dsegE = (float *)(ws + pl.dseg);
    a.acc = (float *)(ws + (a.rep > 1 ? pl.acc : pl.rec));
    a.save = kSuper;
    a.save_per = pl.supers_per;
    a.dg = dg;
    a.dbeta = dbeta;
    hipStream_t st = (hipStream_t)stream;
    const bool bf = p->in_dtype == PGF_BF16;
    if (p->clear_rest) {
        Rest rest{};
        if (p->clear_rest == 1) {
            rest.add(a.dq, a.Hk, a.dk * (int)e, (int)e);
            rest.add(a.dk_, a.Hk, a.dk * (int)e, (int)e);
            rest.add(a.dv_, a.Hv, a.dv * (int)e, (int)e);
        }
        rest.add(View{dg, 0, pl.L, 1}, a.Hv, 4, 4);
        rest.add(View{dbeta, 0, pl.L, 1}, a.Hv, 4, 4);
        clear_rest(rest, a, st);
    }
    if (pl.DK == 64) return bf ? grads_t<__bf16, 64>(a, pl, st) : grads_t<float, 64>(a, pl, st);
    return bf ? grads_t<__bf16, 128>(a, pl, st) : grads_t<float, 128>(a, pl, st);
}
