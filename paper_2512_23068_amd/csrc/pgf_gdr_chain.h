// Kernels shared by the scan and the gradients of the gated delta rule: the
// chunks' records and the forward chain (see pgf_gdr.hip for the chunk form).
#pragma once

#include "pgf_gdr.h"

namespace pgf {
namespace gdr {

struct Args {
    View q, k, v, g, beta, o;
    Seqs seqs;
    int64_t chunk_per, seg_per, seg;     // (Seqs::of)
    int Hk, Hv, rep, dk, dv;             // rep: value heads per key head
    float scale;
    char *rec;                           // [chunk slots][Hv] records
    int grads;                           // the records hold T^ too
    const float *S_in;                   // entry states per sequence (NULL = zero), or
    const float *seg_in;                 // per segment
    float *S_out;
    float *segE, *tr, *trT;              // kSegment: end states, transitions, transposed ones (or NULL)
    float *saveS, *saveE;                // kSave: states entering every save-th chunk, E of every chunk
    int64_t save_per; int save;          // slots of kC * save steps of a dense sequence
    int ct, vt;                          // column tiles of a head, value tiles among them
    // gradients
    View go, dq, dk_, dv_;               // dl/do; dl/dq, dl/dk, dl/dv
    const float *dS_out, *dseg_in;       // dl/dS leaving sequences (NULL = zero), or segments
    float *dS_in;                        // dl/dS entering sequences
    float *dsegE;                        // kBackSegment: adjoint at the segments' starts, from zero
    float *saveD, *saveU;                // kBack: adjoint of the state leaving every save chunks, dl/dE of every chunk
    float *acc;                          // sums of dq over value heads
    float *dg, *dbeta;                   // dense [B][Hv][L]
};

// ---------------------------------------------------------------- prep
// One wave per chunk and key head: K K^T and Q K^T once, then T^, TW and TA of
// each of its value heads.  G and its differences are f64: a difference of two
// long sums would lose the decay between neighbours.  T^ by 16 x 16 blocks: the
// diagonal ones by substitution, one column a lane, the third is -T11 (N10 T00)
// on the f32 matrix cores, as are the products of TA.  A decay below e^-200 a
// step is zero in f32, as is e^-200, so -inf (forget everything) is taken as
// -200 and no difference becomes inf - inf.
// Bound by memory: it reads q and k once and writes the records (6 KB a chunk and
// head; 9 KB with T^): 0.54 ms for 131072 steps of 32 heads in f32 (3.0 GB), 46 us
// for 4 x 4096 steps of 16 heads in bf16, where the chain of one head's decays,
// substitution and products is waited for.
constexpr int kPrepWaves = 4;

// Store at a 32-bit offset from a base that is the same for the whole wave.
template <typename V>
__device__ __forceinline__ void put(char *base, uint32_t bytes, const V &x) { *(V *)(base + (size_t)bytes) = x; }

__device__ __forceinline__ floatx4 mfma_f32(float a, float b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

template <typename T, int DK>
__global__ __launch_bounds__(64 * kPrepWaves)
__attribute__((amdgpu_waves_per_eu(sizeof(T) == 4 && DK == 128 ? 3 : 4))) void k_gdr_prep(Args a, int64_t slots) {
    constexpr int P = sizeof(T) == 2 ? 1 : 3, KS = DK / 32;
    struct Lds {
        __align__(16) float L10[16][20];
        // T^: blocks (0,0), (1,0), (1,1); the diagonal ones first hold those of
        // N diag(beta), by column
        __align__(16) float Ti[3][16][20];
        __align__(16) float A[3][16][20];     // A diag(beta)
        __align__(16) double G[32];
        __align__(16) float be[32];
    };
    __shared__ Lds lds[kPrepWaves];
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int lane = threadIdx.x % 64, c = lane % 16, qd = lane / 16;
    Lds &s = lds[w];
    const int64_t item = (int64_t)blockIdx.x * kPrepWaves + w;
    if (item >= slots * a.Hk) return;
    const int64_t slot = item / a.Hk;
    const int hk = (int)(item - slot * a.Hk);
    const Rows r = a.seqs.of(slot, kC, a.chunk_per);
    if (r.unit0 >= r.len) return;
    const int live = (int)uni(r.len - r.unit0 < kC ? r.len - r.unit0 : kC);
    const int64_t t0 = r.lo + r.unit0;

    floatx4 kk[3], qk[3];                // blocks (0,0), (1,0), (1,1)
#pragma unroll
    for (int i = 0; i < 3; ++i) kk[i] = qk[i] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    {
        const Buf kb = make_buf(row_ptr<T>(a.k, r.b, hk, t0), (uint32_t)a.k.st * sizeof(T), live, a.dk * (int)sizeof(T));
        const Buf qb = make_buf(row_ptr<T>(a.q, r.b, hk, t0), (uint32_t)a.q.st * sizeof(T), live, a.dk * (int)sizeof(T));
        Raw8<T> kx[KS][2], qx[KS][2];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                const uint32_t e = 32 * ks + 8 * qd;
                const bool on = (int)e < a.dk;
                kx[ks][m] = load8<T>(kb, on ? (16 * m + c) * kb.st + e * sizeof(T) : kNone, 0);
                qx[ks][m] = load8<T>(qb, on ? (16 * m + c) * qb.st + e * sizeof(T) : kNone, 0);
            }
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            Frag<P> kf[2], qf[2];
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                kf[m] = raw_frag<P>(kx[ks][m]);
                qf[m] = raw_frag<P>(qx[ks][m]);
            }
            kk[0] = mfma_parts<P, P>(kf[0], kf[0], kk[0]);
            kk[1] = mfma_parts<P, P>(kf[1], kf[0], kk[1]);
            kk[2] = mfma_parts<P, P>(kf[1], kf[1], kk[2]);
            qk[0] = mfma_parts<P, P>(qf[0], kf[0], qk[0]);
            qk[1] = mfma_parts<P, P>(qf[1], kf[0], qk[1]);
            qk[2] = mfma_parts<P, P>(qf[1], kf[1], qk[2]);
        }
    }
    const uint32_t rb = rec_bytes(a.grads);
    for (int vh = 0; vh < a.rep; ++vh) {
        const int h = hk * a.rep + vh;
        char *rec = (char *)uni((int64_t)(uintptr_t)(a.rec + (slot * a.Hv + h) * (int64_t)rb));
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
        s.G[t] = G;                      // (the upper lanes repeat the lower ones)
        s.be[t] = be;
        put(rec, rec_eG(a.grads) + 4 * t, expf((float)G));
        wave_lds();
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            const int bm = i > 0, bn = i > 1;
            const double Gs = s.G[16 * bn + c];
            const float bs = s.be[16 * bn + c];
            floatx4 nb;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int row = 4 * qd + j;
                const bool on = bm != bn || row >= c, below = bm != bn || row > c;
                const float dG = (float)(s.G[16 * bm + row] - Gs);
                const float d = expf(on ? dG : 0.0f) * bs;
                s.A[i][row][c] = on ? d * qk[i][j] : 0.0f;
                nb[j] = below ? d * kk[i][j] : 0.0f;
                if (i == 1) s.L10[row][c] = nb[j];
            }
            if (i != 1) *(floatx4 *)&s.Ti[i][c][4 * qd] = nb;
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
                const floatx4 l = *(const floatx4 *)&s.Ti[2 * bd][j][i4];
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (i4 + i > j) tc[i4 + i] = fmaf(-l[i], tc[j], tc[i4 + i]);
            }
            __builtin_amdgcn_sched_barrier(0);     // one column's reads at a time, or all take registers
        }
        wave_lds();
#pragma unroll
        for (int i = 0; i < 16; ++i) s.Ti[2 * bd][i][c] = tc[i];
        wave_lds();
        floatx4 x = {0.0f, 0.0f, 0.0f, 0.0f}, t10 = x;
#pragma unroll
        for (int j = 0; j < 4; ++j)      // N10 T00; contraction index 4 j + qd
            x = mfma_f32(s.L10[c][4 * j + qd], s.Ti[0][4 * j + qd][c], x);
#pragma unroll
        for (int j = 0; j < 4; ++j)      // T11 x; contraction index 4 qd + j, as x lies
            t10 = mfma_f32(s.Ti[2][c][4 * qd + j], x[j], t10);
#pragma unroll
        for (int j = 0; j < 4; ++j) s.Ti[1][4 * qd + j][c] = -t10[j];
        wave_lds();
        // TA by transposed products, so that a lane receives four columns of a
        // row: row c, columns 4 qd .. 4 qd + 3 of each block
        floatx4 ta[3];
#pragma unroll
        for (int i = 0; i < 3; ++i) ta[i] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int k = 4 * j + qd;
            const float a00 = s.A[0][c][k], a10 = s.A[1][c][k], a11 = s.A[2][c][k];
            const float t00 = s.Ti[0][k][c], t10_ = s.Ti[1][k][c], t11 = s.Ti[2][k][c];
            ta[0] = mfma_f32(t00, a00, ta[0]);
            ta[1] = mfma_f32(t00, a10, ta[1]);
            ta[1] = mfma_f32(t10_, a11, ta[1]);
            ta[2] = mfma_f32(t11, a11, ta[2]);
        }
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            const int row = 16 * (i > 0) + c;
            const uint32_t at = i * kTile + (4 * c + qd) * 16;
            const floatx4 tr = *(const floatx4 *)&s.Ti[i][c][4 * qd];
            const float ob = expf((float)(Gend - s.G[row])) * s.be[row];
            put(rec, at, floatx4{tr[0] * ob, tr[1] * ob, tr[2] * ob, tr[3] * ob});
            put(rec, kMat + at, ta[i]);
            if (a.grads) put(rec, 2 * kMat + at, tr);
        }
    }
}

// ---------------------------------------------------------------- chain
// A wave owns 16 columns of the state of one head, all its keys, in
// accumulators, and takes its segment chunk by chunk; the waves of a block
// share the chunk's keys, queries, TW and TA in LDS.  Every product contracts
// over the rows of the wave's own last result, which lies as the operand it is
// needed as (see mfma), so nothing crosses waves but the staged chunk; the
// next one is loaded into registers meanwhile.
// Bound by issue where two waves share a SIMD: at 128 x 128 in bf16 a wave's chunk is
// 96 matrix instructions of 16 cycles and about 300 vector ones of 2.4, of which half
// take S and X apart, and both need 3 us a chunk.  A wave that has its SIMD to itself
// waits for its own last products instead: 2 us a chunk, or 1.9 with half of the work
// (HS = 2), of which it issues for 1.1 (matrix cores 20 % busy).  4 x 4096 steps of 16
// heads take 232 us (of 277 with the records), 131072 steps of 32 heads of 64 x 64 in
// f32 1.1 ms as kOut, there at the memory's rate (5.1 GB).  32 steps a chunk: a longer
// one has fewer splits of S a step, and longer products with T^.
//   kOut      outputs, from the true entry state
//   kSegment  zero-start end state of the segment (value columns) and its
//             transition (columns of the identity, v = 0)
//   kSave     for the gradients: E of every chunk and the state entering every
//             save-th one
enum Mode { kOut, kSegment, kSave, kBack, kBackSegment };

// Place of M[row][key] in a segment's transition: as the carry's lanes take it, each
// of their loads 1 KB in a piece.
template <int DK>
__device__ __forceinline__ constexpr uint32_t tr_at(int row, int key) {
    return (uint32_t)((((row / 16 * (DK / 32) + key / 32) * 2 + key % 8 / 4) * 64 + key % 32 / 8 * 16 + row % 16) * 4 + key % 4);
}

template <typename T, int DK, int MODE>
struct Chunk {
    static constexpr int P = sizeof(T) == 2 ? 1 : 3;      // parts of q and k
    static constexpr bool HAS_Q = MODE != kSegment && MODE != kSave;
    static constexpr int NI = MODE == kSegment ? 3 : 6;   // images: TW, then TA (kSave: T^)
    __align__(16) char K[P][32 * DK * 2];
    __align__(16) char Q[HAS_Q ? P : 1][HAS_Q ? 32 * DK * 2 : 16];
    __align__(16) char M[NI][kImg];
    __align__(16) float eG[32];
};

// HS = 2: two waves share a column tile, each with half of the keys; they add
// their parts of K S and Q S through LDS and both go on from the sum, each
// updating its keys and writing half the outputs.  A fifth more work for half the
// chain: taken up to as many tiles as leave every SIMD at most one such wave (16
// heads of 128 x 128, 2048 steps, us with one wave a tile and with two: 512 tiles
// 166 and 143, 768 tiles 173 and 195, 1024 tiles 178 and 202).
template <typename T, int DK, int MODE, int HS>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void k_gdr_chain(Args a, uint32_t n_items) {
    using Ck = Chunk<T, DK, MODE>;
    constexpr int P = Ck::P, NI = Ck::NI;
    constexpr bool OUT = MODE == kOut;
    constexpr int NT = 256, TB = 4 / HS;           // threads, column tiles
    constexpr int KS = DK / 32 / HS, KT = DK / 16 / HS;    // of this wave's keys
    constexpr int UNITS = 32 * DK / 8;             // 8-key units of K (and of Q)
    constexpr int KU = (UNITS + NT - 1) / NT;      // those a thread stages
    constexpr int NM = MODE == kSegment ? 1 : 2, MU = (3 * NM + 3) / 4;    // matrices, and tiles of them a wave stages
    // Two chunks in LDS where a CU still holds two blocks (one barrier a chunk).
    constexpr int NB = sizeof(Ck) <= 40960 ? 2 : 1;
    __shared__ Ck lds[NB];
    __shared__ floatx4 sEx[HS > 1 ? HS : 1][HS > 1 ? TB : 1][4][HS > 1 ? 64 : 1];      // [half][tile][K S, Q S][lane]
    const int tid = threadIdx.x, lane = tid % 64, c = lane % 16, qd = lane / 16;
    const int wv = __builtin_amdgcn_readfirstlane(tid / 64), w = wv % TB, hh = wv / TB;
    const int cb = (a.ct + TB - 1) / TB;           // blocks of a head
    const uint32_t item = xcd_item(blockIdx.x, (uint32_t)(cb * a.rep));
    if (item >= n_items) return;
    const int64_t sh = item / cb;
    const int tile = (int)(item - sh * cb) * TB + w;
    const int64_t slot = sh / a.Hv;
    const int h = (int)(sh - slot * a.Hv), hk = h / a.rep;
    const Rows r = a.seqs.of(slot, a.seg ? a.seg : a.seqs.L + 1, a.seg_per);
    // A slot behind its sequence's end has no steps; a sequence of none still
    // hands its state on (its first slot).
    if (r.unit0 > 0 && r.unit0 >= r.len) return;   // uniform over the block
    int64_t n = uni(r.len - r.unit0);
    if (a.seg && n > a.seg) n = a.seg;
    const bool last = r.unit0 + n >= r.len;
    // Nothing follows the last segment; the adjoint passes through its transition
    // to all but the first.
    if (MODE == kSegment && last && (!a.grads || r.unit0 == 0)) return;
    const bool value = tile < a.vt, mine = tile < a.ct;
    const int col = (value ? tile : tile - a.vt) * 16 + c;
    const bool live_col = mine && (value ? col < a.dv : col < a.dk);
    const int chunks = (int)((n + kC - 1) / kC);
    const int64_t t0 = r.lo + r.unit0;
    const int64_t slot0 = uni(a.seqs.slot0(r.n, kC, a.chunk_per) + r.unit0 / kC);

    const int64_t save0 =
        MODE == kSave ? uni(a.seqs.slot0(r.n, kC * a.save, a.save_per) + r.unit0 / (kC * a.save)) : 0;

    // S[kt][j]: key key0(kt) + j of this lane's column
    auto key0 = [&](int kt) { return 32 * (hh * KS + kt / 2) + 8 * qd + 4 * (kt & 1); };
    floatx4 S[KT];
    // States through buffers: lanes and keys without a place read zero and write
    // nothing, and a lane keeps one offset for all its keys.
    const uint32_t est = (uint32_t)a.dv * 4, so = live_col ? (uint32_t)((32 * hh * KS + 8 * qd) * a.dv + col) * 4u : kNone;
    auto state = [&](const float *p) {
        return Buf{__builtin_amdgcn_make_buffer_rsrc((void *)uni((int64_t)(uintptr_t)p), 0, a.dk * a.dv * 4, 0x00020000), est};
    };
    auto place = [&](int kt, int j) { return (uint32_t)(32 * (kt / 2) + 4 * (kt & 1) + j) * est; };
    {
        const float *in = MODE == kSegment ? nullptr : a.seg_in && r.len ? a.seg_in + (slot * a.Hv + h) * a.dk * a.dv
                          : a.S_in ? a.S_in + (r.n * a.Hv + h) * a.dk * a.dv : nullptr;
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) S[kt] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
        if (in) {
            const Buf ib = state(in);
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                for (int j = 0; j < 4; ++j) S[kt][j] = raw_f<float>(load1<float>(ib, so, place(kt, j)));
        }
        if (MODE == kSegment && !value) {
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                for (int j = 0; j < 4; ++j) S[kt][j] = key0(kt) + j == col ? 1.0f : 0.0f;
        }
    }
    auto store_state = [&](float *out) {
        const Buf ob = state(out);
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int j = 0; j < 4; ++j) store1<float>(ob, so, place(kt, j), S[kt][j]);
    };

    // What this thread stages of a chunk.  Rows behind the sequence's end have a
    // beta of zero in the record, so they write nothing, whatever is read there
    // (zero, or where rows overlap, of the last one).
    Raw8<T> rk[KU], rq[OUT ? KU : 1];
    uintx4 rm[MU];
    float reG;
    uint32_t rv[2][4];
    const T *kp = row_ptr<T>(a.k, r.b, hk, t0), *qp = row_ptr<T>(a.q, r.b, hk, t0), *vp = row_ptr<T>(a.v, r.b, h, t0),
            *op = row_ptr<T>(a.o, r.b, h, t0);
    const uint32_t vst = (uint32_t)a.v.st * sizeof(T), ost = (uint32_t)a.o.st * sizeof(T);
    const uint32_t vo = live_col && value ? 4 * qd * vst + col * (uint32_t)sizeof(T) : kNone;
    const uint32_t oo = live_col ? 4 * qd * ost + col * (uint32_t)sizeof(T) : kNone;
    const uint32_t kst = (uint32_t)a.k.st * sizeof(T), qst = (uint32_t)a.q.st * sizeof(T);
    const uint32_t rb = rec_bytes(a.grads);
    uint32_t ko[KU], qo[KU];
#pragma unroll
    for (int i = 0; i < KU; ++i) {
        const int u = tid + NT * i, t = u / (DK / 8), e = u % (DK / 8) * 8;
        const bool on = e < a.dk && u < UNITS;
        ko[i] = on ? t * kst + e * (uint32_t)sizeof(T) : kNone;
        qo[i] = on ? t * qst + e * (uint32_t)sizeof(T) : kNone;
    }
    auto live_rows = [&](int ch) {
        const int64_t left = n - (int64_t)ch * kC;
        return (int)(left < kC ? left : kC);
    };
    auto fetch = [&](int ch) {
        const int live = live_rows(ch);
        const Buf kb = make_buf(kp + (int64_t)ch * kC * a.k.st, kst, live, a.dk * (int)sizeof(T));
        const Buf qb = make_buf(qp + (int64_t)ch * kC * a.q.st, qst, live, a.dk * (int)sizeof(T));
        const Buf vb = make_buf(vp + (int64_t)ch * kC * a.v.st, vst, live, a.dv * (int)sizeof(T));
#pragma unroll
        for (int i = 0; i < KU; ++i) {
            rk[i] = load8<T>(kb, ko[i], 0);
            if constexpr (OUT) rq[i] = load8<T>(qb, qo[i], 0);
        }
        const char *rec = a.rec + ((slot0 + ch) * a.Hv + h) * (int64_t)rb;
#pragma unroll
        for (int i = 0; i < MU; ++i) {
            const int t = wv + 4 * i < 3 * NM ? wv + 4 * i : 0;        // (none: the first again)
            rm[i] = *(const uintx4 *)(rec + (t + (MODE == kSave && t >= 3 ? 3 : 0)) * kTile + 16u * lane);
        }
        reG = *(const float *)(rec + rec_eG(a.grads) + 4 * (tid % 32));
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int j = 0; j < 4; ++j) rv[m][j] = load1<T>(vb, vo, (16 * m + j) * vst);
    };
    auto stage = [&](Ck &s) {
#pragma unroll
        for (int i = 0; i < KU; ++i) {
            const int u = tid + NT * i, t = u / (DK / 8);
            if (64 * wv + NT * i >= UNITS) continue;
            const uint32_t at = unit_off<DK>(t, u % (DK / 8));
            const Frag<P> f = raw_frag<P>(rk[i]);
#pragma unroll
            for (int p = 0; p < P; ++p) *(bf16x8 *)&s.K[p][at] = f.p[p];
            if constexpr (OUT) {
                const Frag<P> y = raw_frag<P>(rq[i]);
#pragma unroll
                for (int p = 0; p < P; ++p) *(bf16x8 *)&s.Q[p][at] = y.p[p];
            }
        }
#pragma unroll
        for (int i = 0; i < MU; ++i) {
            const int t = wv + 4 * i;
            if (t < 3) put_tile<3>(s.M, t, rm[i]);
            else if (t < 3 * NM) put_tile<3>(s.M + NI - 3, t - 3, rm[i]);
        }
        if (tid < 32) s.eG[tid] = reG;
    };

    if (chunks > 0) {
        fetch(0);
#pragma unroll
        for (int i = 0; i < NB; ++i) zero_tile<NI, NT>(lds[i].M, tid);
        stage(lds[0]);
        lds_barrier();
    }
    for (int ch = 0; ch < chunks; ++ch) {
        if constexpr (MODE == kSave)
            if (mine && ch % a.save == 0)
                store_state(a.saveS + ((save0 + ch / a.save) * a.Hv + h) * a.dk * a.dv);
        float vv[2][4];
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int j = 0; j < 4; ++j) vv[m][j] = raw_f<T>(rv[m][j]);
        const Ck &s = lds[NB == 2 ? ch & 1 : 0];
        fetch(ch + 1 < chunks ? ch + 1 : ch);      // (the last chunk again rather than a branch)
        if (HS > 1 || mine) {                      // (waves that share barriers go through the motions)
            // Operands are read a step ahead of their products: left to
            // itself the compiler reads each where it is needed and waits.
            floatx4 kS[2], qS[2];
#pragma unroll
            for (int m = 0; m < 2; ++m) kS[m] = qS[m] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
            Frag<P> kf[2][2], qf[2][2];
            auto read_kq = [&](int ks) {
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int p = 0; p < P; ++p) {
                        const uint32_t at = unit_off<DK>(16 * m + c, 4 * (hh * KS + ks) + qd);
                        kf[ks & 1][m].p[p] = *(const bf16x8 *)&s.K[p][at];
                        if constexpr (OUT) qf[ks & 1][m].p[p] = *(const bf16x8 *)&s.Q[p][at];
                    }
            };
            Frag<3> tf[2];
            floatx4 eG[2];
            read_kq(0);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                if (ks + 1 < KS) read_kq(ks + 1);
                else {
#pragma unroll
                    for (int m = 0; m < 2; ++m) {
#pragma unroll
                        for (int p = 0; p < 3; ++p)
                            tf[m].p[p] = *(const bf16x8 *)&s.M[p][unit_off<32>(16 * m + c, qd)];
                        eG[m] = *(const floatx4 *)&s.eG[16 * m + 4 * qd];
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
                const Frag<3> sp = to_frag<3>(S[2 * ks], S[2 * ks + 1]);
                mfma_parts2<P, 3>(kf[ks & 1], sp, kS);
                if constexpr (OUT) mfma_parts2<P, 3>(qf[ks & 1], sp, qS);
                __builtin_amdgcn_sched_barrier(0);
            }
            if constexpr (HS > 1) {
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    sEx[hh][w][m][lane] = kS[m];
                    if constexpr (OUT) sEx[hh][w][2 + m][lane] = qS[m];
                }
                lds_barrier();
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    kS[m] = sEx[0][w][m][lane] + sEx[1][w][m][lane];
                    if constexpr (OUT) qS[m] = sEx[0][w][2 + m][lane] + sEx[1][w][2 + m][lane];
                }
            }
            floatx4 X[2];
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    X[m][j] = fmaf(-eG[m][j], kS[m][j], vv[m][j]);
                    if constexpr (OUT) qS[m][j] *= eG[m][j];
                }
            const Frag<3> xp = to_frag<3>(X[0], X[1]);
            constexpr int GK = P == 1 && KT >= 4 ? 4 : 2;     // key tiles read at a time
            Frag<P> ktf[2][GK];
            auto read_kt = [&](int g) {
#pragma unroll
                for (int i = 0; i < GK; ++i) {
                    const int kt = hh * KT + g * GK + i, row = 4 * qd + c / 4;
#pragma unroll
                    for (int p = 0; p < P; ++p) {
                        const char *k0 = &s.K[p][unit_off<DK>(row, 4 * (kt / 2) + c % 4) + 8 * (kt & 1)];
                        const char *k1 = &s.K[p][unit_off<DK>(16 + row, 4 * (kt / 2) + c % 4) + 8 * (kt & 1)];
                        ktf[g & 1][i].p[p] = __builtin_shufflevector(read_tr(k0), read_tr(k1), 0, 1, 2, 3, 4, 5, 6, 7);
                    }
                }
            };
            read_kt(0);
            const float end = s.eG[31];
            __builtin_amdgcn_sched_barrier(0);
            floatx4 W[2] = {};
            mfma_parts2<3, 3>(tf, xp, W);
            const Frag<3> wp = to_frag<3>(W[0], W[1]);
            Frag<3> af[2];
            if constexpr (MODE != kSegment) {
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int p = 0; p < 3; ++p)
                        af[m].p[p] = *(const bf16x8 *)&s.M[3 + p][unit_off<32>(16 * m + c, qd)];
            }
#pragma unroll
            for (int g = 0; g < KT / GK; ++g) {
                if (g + 1 < KT / GK) read_kt(g + 1);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < GK; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) S[g * GK + i][j] *= end;
                // part by part over the tiles, so that no product waits for the last one
#pragma unroll
                for (int sum = 2; sum >= 0; --sum)
#pragma unroll
                    for (int p = 0; p < P; ++p)
                        if (sum - p >= 0)
#pragma unroll
                            for (int i = 0; i < GK; ++i)
                                S[g * GK + i] = mfma(ktf[g & 1][i].p[p], wp.p[sum - p], S[g * GK + i]);
                __builtin_amdgcn_sched_barrier(0);
            }
            if constexpr (OUT) {
                const Buf ob = make_buf(op + (int64_t)ch * kC * a.o.st, ost, live_rows(ch), a.dv * (int)sizeof(T));
                if constexpr (HS > 1) {            // (rows 16 hh ..)
                    const floatx4 o = mfma_parts<3, 3>(hh ? af[1] : af[0], xp, hh ? qS[1] : qS[0]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) store1<T>(ob, oo, (16 * hh + j) * ost, o[j] * a.scale);
                } else {
                    mfma_parts2<3, 3>(af, xp, qS);
#pragma unroll
                    for (int m = 0; m < 2; ++m)
#pragma unroll
                        for (int j = 0; j < 4; ++j) store1<T>(ob, oo, (16 * m + j) * ost, qS[m][j] * a.scale);
                }
            }
            if constexpr (MODE == kSave) {
                float *eb = a.saveE + ((slot0 + ch) * a.Hv + h) * (int64_t)(kC * a.dv);
                floatx4 e[2] = {};
                mfma_parts2<3, 3>(af, xp, e);
                const Buf sb{__builtin_amdgcn_make_buffer_rsrc((void *)uni((int64_t)(uintptr_t)eb), 0, kC * a.dv * 4, 0x00020000), est};
                const uint32_t eo = live_col ? (uint32_t)(4 * qd * a.dv + col) * 4u : kNone;
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int j = 0; j < 4; ++j) store1<float>(sb, eo, (16 * m + j) * est, e[m][j]);
            }
        }
        if constexpr (NB == 1) lds_barrier();
        stage(lds[NB == 2 ? (ch + 1) & 1 : 0]);
        lds_barrier();
    }
    if (!mine) return;
    if constexpr (MODE == kSegment) {
        if (value) store_state(a.segE + (slot * a.Hv + h) * a.dk * a.dv);
        else if (live_col) {
            const int64_t at = (slot * a.Hv + h) * DK * DK;
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
                if (key0(kt) < a.dk) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) a.tr[at + tr_at<DK>(key0(kt) + j, col)] = S[kt][j];
                    if (a.trT) *(floatx4 *)(a.trT + at + tr_at<DK>(col, key0(kt))) = S[kt];
                }
        }
    } else if (a.S_out && last) store_state(a.S_out + (r.n * a.Hv + h) * a.dk * a.dv);
}

// ---------------------------------------------------------------- carry
// The state entering each segment of a sequence, one after the other:
// S <- M S + E with the segments' transitions M and zero-start end states E
// (E's place receives the entry state).  BACK: the adjoint leaving each, from
// the last to the first, with M transposed.  A block has 16 value columns of a
// head; its DK / 16 waves share the keys and pass the state's parts through LDS.
// 1.4 us a segment at 128 x 128 (32 segments of 4 heads 43 us): its products wait
// for the last segment's, and three segments are loaded ahead of them.  A block
// reads 64 KB a segment, a thousand cycles of its CU's path to the cache where each
// load takes whole lines (tr_at); rows as they are took 67 us.
template <int DK, bool BACK>
__device__ __forceinline__ void carry(const Args &a, int64_t n, int h, int tile, char (*sS)[16 * DK * 2]) {
    constexpr int KS = DK / 32, D = 3;             // segments loaded ahead
    const int tid = threadIdx.x, lane = tid % 64, c = lane % 16, qd = lane / 16;
    const int w = __builtin_amdgcn_readfirstlane(tid / 64);
    const int64_t slot0 = uni(a.seqs.slot0(n, a.seg, a.seg_per));
    const int64_t len = a.seqs.cu ? (a.seqs.bound(n + 1) > a.seqs.bound(n) ? a.seqs.bound(n + 1) - a.seqs.bound(n) : 0) : a.seqs.L;
    const int G = (int)uni((len + a.seg - 1) / a.seg);
    if (G == 0) return;
    const int col = 16 * tile + c, key = 16 * w + 4 * qd, row = 16 * w + c;
    const int64_t cell = a.dk * a.dv;
    const float *init = BACK ? a.dS_out : a.S_in;
    // segment g's arrays: `step` segments of all heads apart, from the first one taken
    const int64_t first = (slot0 + (BACK ? G - 1 : 0)) * a.Hv + h;
    const int64_t dE = (BACK ? -1 : 1) * (int64_t)a.Hv * cell, dM = (BACK ? -1 : 1) * (int64_t)a.Hv * (DK * DK);
    float *E = (float *)uni((int64_t)(uintptr_t)((BACK ? a.dsegE : a.segE) + first * cell));
    const float *M = (const float *)uni((int64_t)(uintptr_t)((BACK ? a.trT : a.tr) + first * (DK * DK)));
    const uint32_t est = a.dv * 4, ebytes = a.dk * est;
    const uint32_t so = col < a.dv && key < a.dk ? (uint32_t)(key * a.dv + col) * 4u : kNone;    // this lane's four keys
    uint32_t mo[KS];                               // its row of M
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
        mo[ks] = row < a.dk && 32 * ks + 8 * qd < a.dk ? (uint32_t)((w * KS + ks) * 128 + lane) * 16u : kNone;
    auto state = [&](const float *p) { return Buf{__builtin_amdgcn_make_buffer_rsrc((void *)p, 0, (int)ebytes, 0x00020000), est}; };
    floatx4 S = {0.0f, 0.0f, 0.0f, 0.0f}, es[D];
    Raw8<float> ms[D][KS];
    auto fetch = [&](int g, floatx4 &e, Raw8<float> (&m)[KS]) {
        g = g < G ? g : G - 1;
        const Buf eb = state(E + g * dE);
        const Buf mb{__builtin_amdgcn_make_buffer_rsrc((void *)(M + g * dM), 0, DK * DK * 4, 0x00020000), DK * 4};
#pragma unroll
        for (int j = 0; j < 4; ++j) e[j] = raw_f<float>(load1<float>(eb, so, j * est));
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            m[ks].x = load8<__bf16>(mb, mo[ks], 0).x;
            m[ks].y = load8<__bf16>(mb, mo[ks], 1024).x;
        }
    };
    if (init) {
        const Buf ib = state((const float *)uni((int64_t)(uintptr_t)(init + (n * a.Hv + h) * cell)));
#pragma unroll
        for (int j = 0; j < 4; ++j) S[j] = raw_f<float>(load1<float>(ib, so, j * est));
    }
#pragma unroll
    for (int u = 0; u < D; ++u) fetch(u, es[u], ms[u]);
    auto step = [&](int g, floatx4 &e, Raw8<float> (&m)[KS]) {
        char *buf = &sS[3 * (g & 1)][0];
        bf16x4 x[3];
        split4<3>(S, x);
#pragma unroll
        for (int p = 0; p < 3; ++p) *(bf16x4 *)&buf[p * 16 * DK * 2 + unit_off<DK>(c, key / 8) + 2 * (key & 4)] = x[p];
        const Buf eb = state(E + g * dE);
#pragma unroll
        for (int j = 0; j < 4; ++j) store1<float>(eb, so, j * est, S[j]);
        floatx4 acc[2] = {e, {0.0f, 0.0f, 0.0f, 0.0f}};
        Frag<3> mf[KS];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) mf[ks] = raw_frag<3>(m[ks]);
        fetch(g + D, e, m);
        lds_barrier();
        Frag<3> sf[2];
        auto read_s = [&](int ks) {
#pragma unroll
            for (int p = 0; p < 3; ++p) sf[ks & 1].p[p] = *(const bf16x8 *)&buf[p * 16 * DK * 2 + unit_off<DK>(c, 4 * ks + qd)];
        };
        read_s(0);
        // two sums in turn: a product waits for the last one of its sum
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            if (ks + 1 < KS) read_s(ks + 1);
            __builtin_amdgcn_sched_barrier(0);
            int n = 0;
#pragma unroll
            for (int sum = 2; sum >= 0; --sum)
#pragma unroll
                for (int i = 0; i <= sum; ++i, ++n) acc[n & 1] = mfma(mf[ks].p[i], sf[ks & 1].p[sum - i], acc[n & 1]);
        }
        S = acc[0] + acc[1];
    };
    int g0 = 0;
    for (; g0 + D <= G; g0 += D)       // (no condition between the steps: behind one, all loads would be waited for)
#pragma unroll
        for (int u = 0; u < D; ++u) step(g0 + u, es[u], ms[u]);
#pragma unroll
    for (int u = 0; u < D - 1; ++u)
        if (g0 + u < G) step(g0 + u, es[u], ms[u]);
}

// BOTH: the adjoint's carry beside the state's (blockIdx.y).
template <int DK, bool BOTH>
__global__ __launch_bounds__(4 * DK) void k_gdr_carry(Args a) {
    __shared__ __align__(16) char sS[6][16 * DK * 2];      // two states of three parts, by column
    const uint32_t item = xcd_item(blockIdx.x, (uint32_t)a.vt);      // (the tiles of a head read the same M)
    const int64_t nh = item / (uint32_t)a.vt;
    const int tile = (int)(item - nh * a.vt);
    const int64_t n = nh / a.Hv;
    const int h = (int)(nh - n * a.Hv);
    if (n >= a.seqs.n) return;
    if (BOTH && blockIdx.y) carry<DK, true>(a, n, h, tile, sS);
    else carry<DK, false>(a, n, h, tile, sS);
}

// ---------------------------------------------------------------- rows of no sequence
// Zeroes them (packed sequences follow each other: those before the first and
// behind the last) in up to five arrays of rows; one block per 64 rows and array.
struct Rest {
    View v[5];
    int H[5], words[5], esize[5];        // heads, 4-byte words of a row, bytes of an element
    int n = 0;
    void add(const View &x, int heads, int row_bytes, int es) {
        v[n] = x;
        H[n] = heads;
        words[n] = row_bytes / 4;
        esize[n++] = es;
    }
};

template <typename I>              // (a template only so that both files may hold it)
__global__ __launch_bounds__(256) void k_gdr_rest(const Rest a, const Seqs seqs) {
    const int x = blockIdx.y, words = a.words[x];
    const int64_t lo = seqs.bound(0), hi = seqs.bound(seqs.n);
    const int64_t t0 = (int64_t)blockIdx.x * 64;
    const int64_t top = t0 + 64 < seqs.L ? t0 + 64 : seqs.L;
    if (t0 >= lo && top <= hi) return;
    const View v = a.v[x];
    for (int64_t t = t0; t < top; ++t) {
        if (t >= lo && t < hi) continue;
        for (int i = threadIdx.x; i < a.H[x] * words; i += 256) {
            const int h = i / words;
            *((uint32_t *)((char *)v.p + ((int64_t)h * v.sh + t * v.st) * a.esize[x]) + (i - h * words)) = 0u;
        }
    }
}

inline void clear_rest(const Rest &r, const Args &a, hipStream_t st) {
    if (!a.seqs.cu || !a.seqs.L) return;
    hipLaunchKernelGGL((k_gdr_rest<int>), dim3((unsigned)((a.seqs.L + 63) / 64), r.n), dim3(256), 0, st, r,
                       a.seqs);
}

}  // namespace gdr
}  // namespace pgf
