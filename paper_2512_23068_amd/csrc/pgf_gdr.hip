// libpgf: the gated delta rule for gfx950: scan over whole sequences and single
// steps on a pool of states.
//
// Chunk form (C = 32 steps; G the sum of g within the chunk up to and including
// a step, S the state entering it):
//   R = diag(beta) (V - e^G K S)                                     [C x dv]
//   V' = T R,  T = (I + tril(diag(beta) (e^{G_t - G_s} * K K^T), -1))^-1
//   O = scale (e^G Q S + A V'),  A = tril(e^{G_t - G_s} * Q K^T)
//   S' = e^{G_C} S + K^T (e^{G_C - G} V')
// V' are the writes u of the steps, so the chunk ends where the steps do.
//
//   k_gdr_prep    per chunk and head: A, T and the decays (no dependence
//                 between chunks)
//   k_gdr_chain   per head and 16 value columns a wave: the chain over chunks
//   k_gdr_carry   composes segments of chunks where sequences are cut
//   k_gdr_step    single steps
//
// Why chunks of 32: the product of T with R is one contraction of the
// 16x16x32 matrix instruction, and a chunk's keys, queries, T and A take 40
// KB of LDS, so that several blocks share a CU.
#include "pgf_gdr.h"
#include "pgf_timing.h"

namespace pgf {
namespace gdr {

struct Args {
    View q, k, v, g, beta, o;
    Seqs seqs;
    int64_t chunk_per, seg_per, seg;     // (Seqs::of)
    int Hk, Hv, rep, dk, dv;             // rep: value heads per key head
    float scale;
    float *rec;                          // [chunk slots][Hv][kRec]
    const float *S_in;                   // entry states per sequence (NULL = zero), or
    const float *seg_in;                 // per segment
    float *S_out;
    float *segE, *tr;                    // k_gdr_chain<false>: end states and transitions
    int ct, vt;                          // column tiles of a head, value tiles among them
};

// ---------------------------------------------------------------- prep
// Store at a 32-bit offset from a base that is the same for the whole wave.
__device__ __forceinline__ void put(float *base, uint32_t i, float x) { *(float *)((char *)base + (size_t)(i * 4u)) = x; }

// One wave per chunk and key head: K K^T and Q K^T once, then T, A and the
// decays of each of its value heads.  G and its differences are f64: a
// difference of two long sums would lose the decay between neighbours.
// T by 16 x 16 blocks: the diagonal ones by forward substitution, one column a
// lane, the third is -T11 (L10 T00) on the f32 matrix cores.
// A decay below e^-200 a step is zero in f32, as is e^-200, so -inf (forget
// everything) is taken as -200 and no difference becomes inf - inf.
constexpr int kPrepWaves = 4;

template <typename T, int DK>
__global__ __launch_bounds__(64 * kPrepWaves) __attribute__((amdgpu_waves_per_eu(4))) void k_gdr_prep(Args a, int64_t slots) {
    constexpr int P = sizeof(T) == 2 ? 1 : 3, KS = DK / 32;
    __shared__ __align__(16) float sD[kPrepWaves][2][16][20];   // diagonal blocks of the triangle, by column
    __shared__ float sL[kPrepWaves][3][16][17];                 // L10, then T00 and T11
    __shared__ double sG[kPrepWaves][32];
    __shared__ __align__(16) float sB[kPrepWaves][32];
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int lane = threadIdx.x % 64, c = lane % 16, qd = lane / 16;
    const int64_t item = (int64_t)blockIdx.x * kPrepWaves + w;
    if (item >= slots * a.Hk) return;
    const int64_t slot = item / a.Hk;
    const int hk = (int)(item - slot * a.Hk);
    const Rows r = a.seqs.of(slot, kC, a.chunk_per);
    if (r.unit0 >= r.len) return;
    const int live = (int)(r.len - r.unit0 < kC ? r.len - r.unit0 : kC);
    const int64_t t0 = r.lo + r.unit0;

    floatx4 kk[3], qk[3];                // blocks (0,0), (1,0), (1,1)
#pragma unroll
    for (int i = 0; i < 3; ++i) kk[i] = qk[i] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        Frag<P> kf[2], qf[2];
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const int t = 16 * m + c;
            const int e = 32 * ks + 8 * qd;            // 8 keys in a row: any order that A and B share
            Vec4<T> x[2] = {zero4<T>(), zero4<T>()}, y[2] = {zero4<T>(), zero4<T>()};
            if (t < live && e < a.dk) {
                const T *kp = a.k.at<const T>(r.b, hk, t0 + t) + e, *qp = a.q.at<const T>(r.b, hk, t0 + t) + e;
                x[0] = load4(kp);
                x[1] = load4(kp + 4);
                y[0] = load4(qp);
                y[1] = load4(qp + 4);
            }
            kf[m] = to_frag<P>(floatx4{to_f(x[0].v[0]), to_f(x[0].v[1]), to_f(x[0].v[2]), to_f(x[0].v[3])},
                               floatx4{to_f(x[1].v[0]), to_f(x[1].v[1]), to_f(x[1].v[2]), to_f(x[1].v[3])});
            qf[m] = to_frag<P>(floatx4{to_f(y[0].v[0]), to_f(y[0].v[1]), to_f(y[0].v[2]), to_f(y[0].v[3])},
                               floatx4{to_f(y[1].v[0]), to_f(y[1].v[1]), to_f(y[1].v[2]), to_f(y[1].v[3])});
        }
        kk[0] = mfma_parts<P, P>(kf[0], kf[0], kk[0]);
        kk[1] = mfma_parts<P, P>(kf[1], kf[0], kk[1]);
        kk[2] = mfma_parts<P, P>(kf[1], kf[1], kk[2]);
        qk[0] = mfma_parts<P, P>(qf[0], kf[0], qk[0]);
        qk[1] = mfma_parts<P, P>(qf[1], kf[0], qk[1]);
        qk[2] = mfma_parts<P, P>(qf[1], kf[1], qk[2]);
    }
    for (int vh = 0; vh < a.rep; ++vh) {
        const int h = hk * a.rep + vh;
        float *rec = a.rec + (slot * a.Hv + h) * kRec;
        const int t = lane % 32;
        float g = 0.0f, be = 0.0f;
        if (t < live) {
            g = *a.g.at<const float>(r.b, h, t0 + t);
            be = *a.beta.at<const float>(r.b, h, t0 + t);
            g = g < -200.0f ? -200.0f : g;
        }
        double G = g;
#pragma unroll
        for (int m = 1; m < 32; m *= 2) {
            const double o = __shfl_up(G, m, 32);
            if (t >= m) G += o;
        }
        const double Gend = __shfl(G, 31, 32);
        wave_lds();
        if (lane < 32) {
            sG[w][t] = G;
            sB[w][t] = be;
            put(rec, kRecRow + t, expf((float)G));
            put(rec, kRecRow + 32 + t, expf((float)(Gend - G)));
            put(rec, kRecRow + 64 + t, be);
        }
        wave_lds();
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            const int bm = i > 0, bn = i > 1;
            const double Gs = sG[w][16 * bn + c];
            const floatx4 bt = *(const floatx4 *)&sB[w][16 * bm + 4 * qd];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int row = 4 * qd + j;
                const bool on = bm != bn || row >= c, below = bm != bn || row > c;
                const float dG = (float)(sG[w][16 * bm + row] - Gs);
                const float d = expf(on ? dG : 0.0f);
                put(rec, kRecA + 256 * i + 16 * row + c, on ? d * qk[i][j] : 0.0f);
                const float l = below ? bt[j] * (d * kk[i][j]) : 0.0f;
                if (i == 1) sL[w][0][row][c] = l;
                else sD[w][bn][c][row] = l;
            }
        }
        wave_lds();
        // column c of diagonal block qd & 1 (the upper lanes repeat the lower
        // ones): once an entry is known it leaves the rows below it
        const int bd = qd & 1;
        float tc[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) tc[i] = i == c ? 1.0f : 0.0f;
#pragma unroll
        for (int j = 0; j < 15; ++j) {
#pragma unroll
            for (int i4 = j / 4 * 4; i4 < 16; i4 += 4) {
                const floatx4 l = *(const floatx4 *)&sD[w][bd][j][i4];
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (i4 + i > j) tc[i4 + i] = fmaf(-l[i], tc[j], tc[i4 + i]);
            }
            __builtin_amdgcn_sched_barrier(0);     // one column's reads at a time, or all take registers
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            sL[w][1 + bd][i][c] = tc[i];
            put(rec, kRecT + 512 * bd + 16 * i + c, tc[i]);
        }
        wave_lds();
        floatx4 x = {0.0f, 0.0f, 0.0f, 0.0f}, t10 = x;
#pragma unroll
        for (int j = 0; j < 4; ++j)      // L10 T00; contraction index 4 j + qd
            x = __builtin_amdgcn_mfma_f32_16x16x4f32(sL[w][0][c][4 * j + qd], sL[w][1][4 * j + qd][c], x, 0, 0, 0);
#pragma unroll
        for (int j = 0; j < 4; ++j)      // T11 x; contraction index 4 qd + j, as x lies
            t10 = __builtin_amdgcn_mfma_f32_16x16x4f32(sL[w][2][c][4 * qd + j], x[j], t10, 0, 0, 0);
#pragma unroll
        for (int j = 0; j < 4; ++j) put(rec, kRecT + 256 + 16 * (4 * qd + j) + c, -t10[j]);
    }
}

// ---------------------------------------------------------------- chain
// A wave owns 16 columns of the state of one head, all its keys, in
// accumulators, and takes its segment chunk by chunk; the four waves of a
// block share the chunk's keys, queries, T and A in LDS.  Every product
// contracts over the rows of the wave's own last result, which lies as the
// operand it is needed as (see mfma), so nothing crosses waves but the staged
// chunk; the next one is loaded into registers meanwhile.
//
// OUT: outputs, from the true entry state.  Otherwise the zero-start end state
// of the segment (value columns) and its transition (columns of the identity,
// v = 0).
template <typename T>
struct Unit { Vec4<T> r[4]; };       // 4 steps x 4 keys

template <typename T, int DK, bool OUT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void k_gdr_chain(Args a, uint32_t n_items) {
    constexpr int P = sizeof(T) == 2 ? 1 : 3;      // parts of q and k
    constexpr int PO = sizeof(T) == 2 ? 2 : 3;     // parts of f32 operands of the output alone
    constexpr int KS = DK / 32, KT = DK / 16;
    constexpr int UNITS = 8 * DK / 4;              // 4 x 4 units of K (and of Q)
    constexpr int NU = (OUT ? 2 : 1) * UNITS / 256 > 0 ? (OUT ? 2 : 1) * UNITS / 256 : 1;
    __shared__ __align__(16) __bf16 sK[P][32][DK + 8];
    __shared__ __align__(16) __bf16 sQ[OUT ? P : 1][OUT ? 32 : 1][OUT ? DK + 8 : 8];
    __shared__ __align__(16) __bf16 sKt[P][DK][40];
    __shared__ __align__(16) __bf16 sT[3][32][40];
    __shared__ __align__(16) __bf16 sA[OUT ? PO : 1][OUT ? 32 : 1][40];
    __shared__ __align__(16) float sRow[3][32];
    const int tid = threadIdx.x, lane = tid % 64, c = lane % 16, qd = lane / 16;
    const int w = __builtin_amdgcn_readfirstlane(tid / 64);
    const int cb = (a.ct + 3) / 4;                 // blocks of a head
    const uint32_t item = xcd_order(blockIdx.x, n_items);
    const int64_t sh = item / cb;
    const int tile = (int)(item - sh * cb) * 4 + w;
    const int64_t slot = sh / a.Hv;
    const int h = (int)(sh - slot * a.Hv), hk = h / a.rep;
    const int64_t unit = a.seg ? a.seg : a.seqs.L + 1;
    const Rows r = a.seqs.of(slot, unit, a.seg_per);
    // A slot behind its sequence's end has no steps; a sequence of none still
    // hands its state on (its first slot).
    if (r.unit0 > 0 && r.unit0 >= r.len) return;   // uniform over the block
    int64_t n = r.len - r.unit0;
    if (a.seg && n > a.seg) n = a.seg;
    const bool last = r.unit0 + n >= r.len;
    const bool value = tile < a.vt, mine = tile < a.ct;
    const int col = (value ? tile : tile - a.vt) * 16 + c;
    const bool live_col = mine && (value ? col < a.dv : col < a.dk);
    const int chunks = (int)((n + kC - 1) / kC);
    const int64_t t0 = r.lo + r.unit0;
    const int64_t slot0 = a.seqs.slot0(r.n, kC, a.chunk_per) + r.unit0 / kC;

    floatx4 S[KT];
    {
        const float *in = OUT ? (a.seg_in ? a.seg_in + (slot * a.Hv + h) * a.dk * a.dv
                                          : a.S_in ? a.S_in + (r.n * a.Hv + h) * a.dk * a.dv : nullptr)
                              : nullptr;
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int key = 16 * kt + 4 * qd + j;
                S[kt][j] = 0.0f;
                if (OUT && in && live_col && key < a.dk) S[kt][j] = in[(int64_t)key * a.dv + col];
                if (!OUT && !value && key == col) S[kt][j] = 1.0f;
            }
    }
    // above the diagonal of T and A
    for (int i = tid; i < 3 * 32 * 40; i += 256) (&sT[0][0][0])[i] = (__bf16)0.0f;
    if constexpr (OUT)
        for (int i = tid; i < PO * 32 * 40; i += 256) (&sA[0][0][0])[i] = (__bf16)0.0f;

    // What this thread stages of a chunk: units of K and Q, float4 of T, A and the rows.
    Unit<T> un[NU];
    floatx4 rt[2];
    float rrow;
    T rv[2][4];
    const int n_rec = OUT ? 384 : 192;             // float4 of T (and A)
    auto fetch = [&](int ch) {
        const int64_t base = t0 + (int64_t)ch * kC;
        const int64_t left = n - (int64_t)ch * kC;
        const int live = (int)(left < kC ? left : kC);
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const int u = tid + 256 * i;
            const bool isq = u >= UNITS;
            const int uu = isq ? u - UNITS : u;
            const int t4 = uu / (DK / 4) * 4, e = uu % (DK / 4) * 4;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                un[i].r[j] = zero4<T>();
                if (t4 + j < live && e < a.dk && (u < UNITS || (OUT && u < 2 * UNITS)))
                    un[i].r[j] = load4((isq ? a.q : a.k).template at<const T>(r.b, hk, base + t4 + j) + e);
            }
        }
        const float *rec = a.rec + ((slot0 + ch) * a.Hv + h) * kRec;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int u = tid + 256 * i;
            if (u < n_rec) rt[i] = *(const floatx4 *)(rec + 4 * u);
        }
        rrow = tid < 96 ? rec[kRecRow + tid] : 0.0f;
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int t = 16 * m + 4 * qd + j;
                rv[m][j] = (T)0.0f;
                if (value && live_col && t < live) rv[m][j] = a.v.at<const T>(r.b, h, base + t)[col];
            }
    };
    auto stage = [&]() {
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const int u = tid + 256 * i;
            const bool isq = u >= UNITS;
            if (!(u < UNITS || (OUT && u < 2 * UNITS))) continue;
            const int uu = isq ? u - UNITS : u;
            const int t4 = uu / (DK / 4) * 4, e = uu % (DK / 4) * 4;
            __bf16 x[4][4][P];
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    if constexpr (P == 1) x[j][m][0] = un[i].r[j].v[m];
                    else split<P>(un[i].r[j].v[m], x[j][m]);
                }
            const int pe = e / 32 * 32 + perm32(e % 32);
#pragma unroll
            for (int p = 0; p < P; ++p) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const bf16x4 y = {x[j][0][p], x[j][1][p], x[j][2][p], x[j][3][p]};
                    if (!isq) *(bf16x4 *)&sK[p][t4 + j][pe] = y;
                    else if constexpr (OUT) *(bf16x4 *)&sQ[p][t4 + j][pe] = y;
                }
                if (!isq) {
#pragma unroll
                    for (int m = 0; m < 4; ++m)
                        *(bf16x4 *)&sKt[p][e + m][perm32(t4)] = bf16x4{x[0][m][p], x[1][m][p], x[2][m][p], x[3][m][p]};
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int u = tid + 256 * i;
            if (u >= n_rec) continue;
            const int blk = u / 64, bi = blk % 3;
            const int row = (bi > 0 ? 16 : 0) + u % 64 / 4, cc = perm32((bi > 1 ? 16 : 0) + u % 4 * 4);
            __bf16 x[4][3];
#pragma unroll
            for (int m = 0; m < 4; ++m) split<3>(rt[i][m], x[m]);
#pragma unroll
            for (int p = 0; p < 3; ++p) {
                const bf16x4 y = {x[0][p], x[1][p], x[2][p], x[3][p]};
                if (blk < 3) *(bf16x4 *)&sT[p][row][cc] = y;
                else if constexpr (OUT) {
                    if (p < PO) *(bf16x4 *)&sA[p][row][cc] = y;
                }
            }
        }
        if (tid < 96) (&sRow[0][0])[tid] = rrow;
    };

    if (chunks > 0) {
        fetch(0);
        lds_barrier();                             // (the zeros)
        stage();
        lds_barrier();
    }
    for (int ch = 0; ch < chunks; ++ch) {
        float vv[2][4];
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int j = 0; j < 4; ++j) vv[m][j] = to_f(rv[m][j]);
        if (ch + 1 < chunks) fetch(ch + 1);
        if (mine) {
            floatx4 kS[2], qS[2];
#pragma unroll
            for (int m = 0; m < 2; ++m) kS[m] = qS[m] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const Frag<3> sp = to_frag<3>(S[2 * ks], S[2 * ks + 1]);
                Frag<PO> so;
#pragma unroll
                for (int p = 0; p < PO; ++p) so.p[p] = sp.p[p];
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    Frag<P> f;
#pragma unroll
                    for (int p = 0; p < P; ++p) f.p[p] = *(const bf16x8 *)&sK[p][16 * m + c][32 * ks + 8 * qd];
                    kS[m] = mfma_parts<P, 3>(f, sp, kS[m]);
                    if constexpr (OUT) {
#pragma unroll
                        for (int p = 0; p < P; ++p) f.p[p] = *(const bf16x8 *)&sQ[p][16 * m + c][32 * ks + 8 * qd];
                        qS[m] = mfma_parts<P, PO>(f, so, qS[m]);
                    }
                }
            }
            floatx4 R[2];
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                const floatx4 eG = *(const floatx4 *)&sRow[0][16 * m + 4 * qd];
                const floatx4 be = *(const floatx4 *)&sRow[2][16 * m + 4 * qd];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    R[m][j] = be[j] * fmaf(-eG[j], kS[m][j], vv[m][j]);
                    if constexpr (OUT) qS[m][j] *= eG[j];
                }
            }
            const Frag<3> rp = to_frag<3>(R[0], R[1]);
            floatx4 U[2];
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                Frag<3> f;
#pragma unroll
                for (int p = 0; p < 3; ++p) f.p[p] = *(const bf16x8 *)&sT[p][16 * m + c][8 * qd];
                U[m] = mfma_parts<3, 3>(f, rp, floatx4{0.0f, 0.0f, 0.0f, 0.0f});
            }
            floatx4 W[2];
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                const floatx4 ou = *(const floatx4 *)&sRow[1][16 * m + 4 * qd];
#pragma unroll
                for (int j = 0; j < 4; ++j) W[m][j] = ou[j] * U[m][j];
            }
            const Frag<3> wp = to_frag<3>(W[0], W[1]);
            const float end = sRow[0][31];
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) {
                Frag<P> f;
#pragma unroll
                for (int p = 0; p < P; ++p) f.p[p] = *(const bf16x8 *)&sKt[p][16 * kt + c][8 * qd];
#pragma unroll
                for (int j = 0; j < 4; ++j) S[kt][j] *= end;
                S[kt] = mfma_parts<P, 3>(f, wp, S[kt]);
            }
            if constexpr (OUT) {
                const Frag<PO> up = to_frag<PO>(U[0], U[1]);
                const int64_t base = t0 + (int64_t)ch * kC;
                const int64_t left = n - (int64_t)ch * kC;
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    Frag<PO> f;
#pragma unroll
                    for (int p = 0; p < PO; ++p) f.p[p] = *(const bf16x8 *)&sA[p][16 * m + c][8 * qd];
                    const floatx4 o = mfma_parts<PO, PO>(f, up, qS[m]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int t = 16 * m + 4 * qd + j;
                        if (live_col && t < left) a.o.at<T>(r.b, h, base + t)[col] = (T)(o[j] * a.scale);
                    }
                }
            }
        }
        if (ch + 1 < chunks) {
            lds_barrier();
            stage();
            lds_barrier();
        }
    }

    if (!live_col) return;
    if constexpr (OUT) {
        if (!a.S_out || !last) return;
        float *out = a.S_out + (r.n * a.Hv + h) * a.dk * a.dv + col;
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int key = 16 * kt + 4 * qd + j;
                if (key < a.dk) out[(int64_t)key * a.dv] = S[kt][j];
            }
    } else {
        const int64_t ld = value ? a.dv : DK;
        float *out = (value ? a.segE + (slot * a.Hv + h) * a.dk * a.dv : a.tr + (slot * a.Hv + h) * DK * DK) + col;
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int key = 16 * kt + 4 * qd + j;
                if (key < a.dk) out[(int64_t)key * ld] = S[kt][j];
            }
    }
}

// ---------------------------------------------------------------- single steps
// A block holds CB value columns of one state in registers: thread (kg, cg)
// has the keys kg + KG i of the columns 4 cg .. 4 cg + 3.  One pass forms S^T k
// and S^T q on the decayed state together (o = S^T q + (k.q) u after the
// write), so a token costs one reduction over the block.  Bound by memory: the
// state is read and written once, whatever the number of steps.
template <typename T, int DK, int CB>
__global__ __launch_bounds__(256) void k_gdr_step(Args a, float *pool, int64_t n_pool, const int32_t *slots, int64_t L,
                                                  uint32_t n_items) {
    constexpr int CG = CB / 4, KG = 256 / CG, KPT = DK / KG;      // keys a thread
    constexpr int WG = 64 / CG;                                  // key groups of a wave
    __shared__ __align__(16) float sKQ[2][DK];
    __shared__ __align__(16) floatx4 sRed[4][2][CG];
    __shared__ float sDot[4];
    __shared__ int sDup;
    const int tid = threadIdx.x, cg = tid % CG, kg = tid / CG;
    const int w = __builtin_amdgcn_readfirstlane(tid / 64), lane = tid % 64;
    const int cb = (a.dv + CB - 1) / CB;
    const uint32_t item = xcd_order(blockIdx.x, n_items);
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
            if (on) {
                T *o = a.o.at<T>(b, h, t) + col;
#pragma unroll
                for (int j = 0; j < 4; ++j) o[j] = (T)0.0f;
            }
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
            const float kx = tid < a.dk ? to_f(a.k.at<const T>(b, hk, t)[tid]) : 0.0f;
            const float qx = tid < a.dk ? to_f(a.q.at<const T>(b, hk, t)[tid]) : 0.0f;
            sKQ[0][tid] = kx;
            sKQ[1][tid] = qx;
            kq = kx * qx;
        }
#pragma unroll
        for (int m = 1; m < 64; m *= 2) kq += __shfl_xor(kq, m, 64);
        if (lane == 0) sDot[w] = kq;
        Vec4<T> v = zero4<T>();
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
        float u[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) u[j] = be * (to_f(v.v[j]) - sk[j]);
#pragma unroll
        for (int i = 0; i < KPT; ++i) {
            const float kx = sKQ[0][kg + KG * i];
#pragma unroll
            for (int j = 0; j < 4; ++j) S[i][j] = fmaf(kx, u[j], S[i][j]);
        }
        if (on && kg == 0) {
            T *o = a.o.at<T>(b, h, t) + col;
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] = (T)(a.scale * fmaf(dot, u[j], sq[j]));
        }
        __syncthreads();
    }
    (void)WG;
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
        const int key = kg + KG * i;
        if (on && key < a.dk) *(floatx4 *)(st + (int64_t)key * a.dv) = S[i];
    }
}

// ---------------------------------------------------------------- dispatch
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
    const uint32_t items = (uint32_t)(pl.seg_slots * pl.Hv * ((a.ct + 3) / 4));
    Timed tm(3, st);
    hipLaunchKernelGGL((k_gdr_chain<T, DK, true>), dim3(items), dim3(256), 0, st, a, items);
    return hipGetLastError() == hipSuccess ? PGF_OK : PGF_ERR_HIP;
}

template <typename T>
int step_t(const Args &a, const Plan &pl, const pgf_gdr_params *p, hipStream_t st) {
    Timed tm(3, st);
    const int64_t bh = pl.B * pl.Hv;
#define PGF_STEP(DK_, CB_)                                                                                         \
    {                                                                                                              \
        const uint32_t items = (uint32_t)(bh * ((pl.dv + CB_ - 1) / CB_));                                         \
        hipLaunchKernelGGL((k_gdr_step<T, DK_, CB_>), dim3(items), dim3(256), 0, st, a, p->S_pool, p->pool,        \
                           p->slots, pl.L, items);                                                                 \
    }
    // 128 columns a block once these fill the GPU, 32 before (four times the
    // blocks, each with a quarter of the state).
    const bool wide = bh * ((pl.dv + 127) / 128) >= 512;
    if (pl.DK == 64) {
        if (wide) PGF_STEP(64, 128) else PGF_STEP(64, 32)
    } else {
        if (wide) PGF_STEP(128, 128) else PGF_STEP(128, 32)
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
    const size_t no = extent(p->o_strides, pl.B, pl.Hv, pl.L, pl.dv, e);
    const size_t ns = (size_t)(pl.nseq * pl.Hv * pl.dk * pl.dv) * 4;
    const struct { const void *p; size_t n; } ins[] = {
        {q, extent(p->q_strides, pl.B, pl.Hk, pl.L, pl.dk, e)}, {k, extent(p->k_strides, pl.B, pl.Hk, pl.L, pl.dk, e)},
        {v, extent(p->v_strides, pl.B, pl.Hv, pl.L, pl.dv, e)}, {g, extent(p->g_strides, pl.B, pl.Hv, pl.L, 1, 4)},
        {beta, extent(p->beta_strides, pl.B, pl.Hv, pl.L, 1, 4)}, {p->S_in, ns}};
    for (const auto &i : ins)
        if (overlaps(o, no, i.p, i.n) || overlaps(p->workspace, pl.total, i.p, i.n)) return PGF_ERR_INVALID_ARG;
    // S_out may be S_in (each state is read before it is written) unless segments read it again.
    for (int i = 0; i < 5; ++i)
        if (overlaps(p->S_out, ns, ins[i].p, ins[i].n)) return PGF_ERR_INVALID_ARG;
    if (overlaps(p->S_out, ns, p->S_in, ns) && p->S_out != p->S_in) return PGF_ERR_INVALID_ARG;
    if (overlaps(o, no, p->S_out, ns) || overlaps(p->workspace, pl.total, o, no) ||
        overlaps(p->workspace, pl.total, p->S_out, ns))
        return PGF_ERR_INVALID_ARG;
    (void)hipGetLastError();
    Args a = make_args(pl, p, q, k, v, g, beta, o);
    char *ws = (char *)p->workspace;
    a.rec = (float *)(ws + pl.rec);
    a.segE = (float *)(ws + pl.segE);
    a.tr = (float *)(ws + pl.tr);
    hipStream_t st = (hipStream_t)stream;
    const bool bf = p->in_dtype == PGF_BF16;
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
    const size_t no = extent(p->o_strides, pl.B, pl.Hv, pl.L, pl.dv, e);
    const size_t ns = (size_t)(p->pool * pl.Hv * pl.dk * pl.dv) * 4;
    const struct { const void *p; size_t n; } ins[] = {
        {q, extent(p->q_strides, pl.B, pl.Hk, pl.L, pl.dk, e)}, {k, extent(p->k_strides, pl.B, pl.Hk, pl.L, pl.dk, e)},
        {v, extent(p->v_strides, pl.B, pl.Hv, pl.L, pl.dv, e)}, {g, extent(p->g_strides, pl.B, pl.Hv, pl.L, 1, 4)},
        {beta, extent(p->beta_strides, pl.B, pl.Hv, pl.L, 1, 4)}, {p->slots, (size_t)pl.B * 4}};
    for (const auto &i : ins)
        if (overlaps(o, no, i.p, i.n) || overlaps(p->S_pool, ns, i.p, i.n)) return PGF_ERR_INVALID_ARG;
    if (overlaps(o, no, p->S_pool, ns)) return PGF_ERR_INVALID_ARG;
    if (pl.L == 0) return PGF_OK;
    (void)hipGetLastError();
    const Args a = make_args(pl, p, q, k, v, g, beta, o);
    return p->in_dtype == PGF_BF16 ? step_t<__bf16>(a, pl, p, (hipStream_t)stream)
                                   : step_t<float>(a, pl, p, (hipStream_t)stream);
}
