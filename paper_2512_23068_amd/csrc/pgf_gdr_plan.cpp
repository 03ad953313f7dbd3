// Host-side planning of the gated delta rule and of the query/key
// preparation (see pgf_gdr_plan.h).
#include "pgf_gdr_plan.h"

#include <algorithm>
#include <cmath>

namespace pgf {

namespace {

constexpr int64_t kMaxItems = int64_t(1) << 30;
constexpr int64_t kMaxHeads = int64_t(1) << 16, kMaxBatch = int64_t(1) << 24, kMaxLen = int64_t(1) << 32;
constexpr int64_t kMaxStride = int64_t(1) << 44;
constexpr int64_t kMaxStep = (int64_t(1) << 24) - 1;      // bytes from step to step
constexpr size_t kMaxTotal = size_t(1) << 46;

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Whether a launch has fewer than 2^32 threads: of more, only the low 32 bits of
// their number run, without an error (2^24 + 1 blocks of 256: one block).
bool fits(int64_t blocks, int64_t threads) { return (double)blocks * (double)threads < 4294967296.0; }

// Strides of an array of rows of `width` elements: not negative, bounded, in
// units of 16 bytes.  An output's rows lie apart: of the indexes that move, in the
// order of their strides, each steps over all that the ones before it span.
bool strides_ok(const int64_t (&s)[3], int64_t unit, bool out, int64_t B, int64_t H, int64_t L, int64_t width) {
    const int64_t n[3] = {B, H, L};
    for (int i = 0; i < 3; ++i)
        if (s[i] < 0 || s[i] > kMaxStride || s[i] % unit) return false;
    // (the array's extent in elements, so that no offset leaves 64 bits)
    if ((double)B * (double)s[0] + (double)H * (double)s[1] + (double)L * (double)s[2] >= 1e17) return false;
    if (!out || L < 1 || (!s[0] && !s[1] && !s[2])) return true;
    int order[3] = {0, 1, 2};
    std::sort(order, order + 3, [&](int x, int y) { return s[x] < s[y]; });
    int64_t span = width;
    for (int i : order) {
        if (n[i] <= 1) continue;
        if (s[i] < span) return false;
        span += (n[i] - 1) * s[i];
    }
    return true;
}

// Adds a section of n * each bytes; false when the workspace would leave any
// sensible size.
bool section(size_t *total, size_t *at, int64_t n, int64_t each) {
    *at = *total;
    const double want = (double)n * (double)each;
    if (want > (double)kMaxTotal) return false;
    *total += ((size_t)n * (size_t)each + 255) / 256 * 256;
    return *total <= kMaxTotal;
}

}  // namespace

void dense_strides(const int64_t (&in)[3], int64_t heads, int64_t L, int64_t width, int64_t (&out)[3]) {
    const bool dense = !in[0] && !in[1] && !in[2];
    out[0] = dense ? heads * L * width : in[0];
    out[1] = dense ? L * width : in[1];
    out[2] = dense || L <= 1 ? width : in[2];
}

size_t extent(const int64_t (&s)[3], int64_t B, int64_t heads, int64_t L, int64_t width, size_t elem) {
    if (B < 1 || heads < 1 || L < 1 || width < 1) return 0;
    int64_t d[3];
    dense_strides(s, heads, L, width, d);
    return (size_t)((B - 1) * d[0] + (heads - 1) * d[1] + (L - 1) * d[2] + width) * elem;
}

bool overlaps(const void *a, size_t na, const void *b, size_t nb) {
    const uintptr_t pa = (uintptr_t)a, pb = (uintptr_t)b;
    return a && b && na && nb && pa < pb + nb && pb < pa + na;
}

bool overlaps(const Arr &a, const Arr &b) {
    if (!overlaps(a.p, a.bytes(), b.p, b.bytes())) return false;
    int64_t x[3], y[3];
    dense_strides(a.s, a.H, a.L, a.width, x);
    dense_strides(b.s, b.H, b.L, b.width, y);
    // Bytes modulo a stride: an index that steps by a multiple of it adds nothing, any
    // other its whole span.  What lies in different places there lies apart.
    const int64_t d = (int64_t)((intptr_t)b.p - (intptr_t)a.p);
    auto span = [](const Arr &r, const int64_t (&s)[3], int64_t period) {
        const int64_t n[3] = {r.B, r.H, r.L}, e = (int64_t)r.elem;
        int64_t bytes = r.width * e;
        for (int i = 0; i < 3; ++i)
            if (s[i] * e % period) bytes += (n[i] - 1) * s[i] * e;
        return bytes;
    };
    const int64_t n[3] = {a.B, a.H, a.L};
    for (int i = 0; i < 3; ++i) {
        const int64_t period = x[i] * (int64_t)a.elem;
        if (n[i] < 2 || period <= 0) continue;
        const int64_t off = (d % period + period) % period;
        if (off >= span(a, x, period) && off + span(b, y, period) <= period) return false;
    }
    return true;
}

namespace gdr {

namespace {

// Time in us of a pass of `waves` waves over `chunks` chunks of 32 steps each, on
// 1024 SIMDs: 2 us a chunk for a wave that has its SIMD to itself, 3 us for two
// that share one; more follow as those end, half evenly, half in whole rounds.
double pass(double waves, double chunks) {
    const double rounds = std::floor(waves / 2048.0), rest = waves - 2048.0 * rounds;
    const double tail = rest <= 0.0 ? 0.0 : rest <= 1024.0 ? 2.0 : 3.0;
    if (rounds < 1.0) return chunks * tail;
    return chunks * 0.5 * (3.0 * rounds + tail + 3.0 * waves / 2048.0);
}

// Steps per segment, 0 = not cut.  A wave takes 16 columns of one head through
// its chunks one after the other, two that share a tile in 1.9 us each (the scan's
// outputs where they are as few as kShareTiles).  Cutting a sequence costs the
// zero-start end states and the transitions (dk more columns, without outputs: 3/4
// of the work a column) on top, the carry, 1.4 us a segment one after the other and
// one block a CU, and two more launches.  Of the lengths below, that of the least
// sum is taken.  Measured, dk = dv = 128, bf16, us: 4 heads of 1024 steps 74 uncut,
// 57 in segments of 256; of 32768 steps 1785 uncut, 337 / 250 / 226 / 263 / 446 in
// segments of 256 / 512 / 1024 / 2048 / 4096; 32 heads of 16384 steps 961 uncut,
// 790 / 639 / 580 / 549 / 639; 4 x 16 heads of 4096 steps 272
// uncut, 284 in segments of 1024.
int64_t default_seg(const Plan &q, bool packed, bool grads) {
    const int64_t unit = kSuper * kC, steps = packed ? q.L : q.B * q.L;
    // Packed lengths are on the device: the longest is taken as four times the mean.
    const int64_t longest = packed ? std::min(q.L, 4 * cdiv(q.L, q.nseq)) : q.L;
    const double vt = (double)(q.Hv * cdiv(q.dv, 16)), kt = (double)(q.Hv * cdiv(q.dk, 16));
    const double tiles = (double)q.nseq * vt;
    double least = std::max(pass(tiles, (double)cdiv(cdiv(steps, q.nseq), kC)), (double)cdiv(longest, kC) * 2.0);
    if (!grads && tiles <= (double)kShareTiles) least *= 0.9;
    int64_t seg = 0;
    for (int64_t n = 4, more = 2; n * unit < longest; n += more) {
        if (n == 4 * more) more *= 2;
        const double chunks = (double)(n * unit / kC), pieces = (double)std::max(cdiv(steps, n * unit), q.nseq);
        const double t = pass(pieces * vt, chunks) + 0.75 * pass(pieces * (vt + kt), chunks) +
                         1.4 * (double)cdiv(longest, n * unit) * std::max(1.0, tiles / 256.0) + 15.0;
        if (t < least) {
            least = t;
            seg = n * unit;
        }
    }
    return seg;
}

}  // namespace

int make_plan(const pgf_gdr_params *p, Plan *out, bool grads, bool step) {
    if (!p || !out) return PGF_ERR_INVALID_ARG;
    Plan q{};
    q.B = p->batch; q.Hk = p->key_heads; q.Hv = p->value_heads; q.L = p->seqlen; q.dk = p->d_key; q.dv = p->d_value;
    if (q.B < 1 || q.Hk < 1 || q.Hv < 1 || q.L < 0 || q.dk < 1 || q.dv < 1 || p->n_seqs < 0) return PGF_ERR_INVALID_ARG;
    if (p->in_dtype != PGF_F32 && p->in_dtype != PGF_BF16) return PGF_ERR_INVALID_ARG;
    if (q.Hv % q.Hk) return PGF_ERR_INVALID_ARG;
    if (q.dk % 8 || q.dk > 128 || q.dv % 8 || q.dv > 4096) return PGF_ERR_UNSUPPORTED;
    if (q.B > kMaxBatch || q.Hv > kMaxHeads || q.L > kMaxLen || p->n_seqs > kMaxBatch) return PGF_ERR_UNSUPPORTED;
    if (p->n_seqs && (q.B != 1 || step)) return PGF_ERR_INVALID_ARG;
    if (p->clear_rest < 0 || p->clear_rest > 2) return PGF_ERR_INVALID_ARG;
    if (p->seg_len < -1 || (p->seg_len > 0 && p->seg_len % (kSuper * kC))) return PGF_ERR_INVALID_ARG;
    const int64_t unit = p->in_dtype == PGF_BF16 ? 8 : 4;
    const struct { const int64_t (&s)[3]; int64_t unit; bool out; int64_t heads, width; } arrays[] = {
        {p->q_strides, unit, false, q.Hk, q.dk}, {p->k_strides, unit, false, q.Hk, q.dk},
        {p->v_strides, unit, false, q.Hv, q.dv}, {p->g_strides, 1, false, q.Hv, 1},
        {p->beta_strides, 1, false, q.Hv, 1}, {p->o_strides, unit, !grads, q.Hv, q.dv},
        {p->dq_strides, unit, grads, q.Hk, q.dk}, {p->dk_strides, unit, grads, q.Hk, q.dk},
        {p->dv_strides, unit, grads, q.Hv, q.dv}};
    for (const auto &a : arrays)
        if (!strides_ok(a.s, a.unit, a.out, q.B, a.heads, q.L, a.width)) return PGF_ERR_INVALID_ARG;
    for (const auto &a : arrays)
        if (q.L > 1 && a.s[2] * (a.unit == 1 ? 4 : 16 / unit) > kMaxStep) return PGF_ERR_UNSUPPORTED;
    if ((double)q.B * (double)q.Hv * (double)q.L * (double)std::max(q.dk, q.dv) > 4e18) return PGF_ERR_UNSUPPORTED;
    q.DK = q.dk <= 64 ? 64 : 128;
    q.nseq = p->n_seqs ? p->n_seqs : q.B;
    // An upper bound of the blocks of one head.
    const int64_t col_blocks = cdiv(q.dv, 16) + q.DK / 16;
    if (step) {
        if (p->pool < 0 || p->pool > kMaxLen) return PGF_ERR_INVALID_ARG;
        if (q.B * q.Hv > kMaxItems / col_blocks) return PGF_ERR_UNSUPPORTED;
        // 32 value columns a block for one or two steps: more blocks have loads in
        // flight (one step of 4096 states of 128 x 128 95 us, with 128 columns a block
        // 94; of 1024 states 24.8 and 26.7).  Further steps wait for each other within
        // a block, and a quarter of the blocks wait a quarter of the time once there is
        // more than the GPU holds (16 steps of 2048 states 247 us, with 128 columns a
        // block 139; of 256 states 44 and 38, 4 steps of 256 states 16 and 16).
        q.step_cols = q.L > 2 && q.B * q.Hv * cdiv(q.dv, 128) >= 256 ? 128 : 32;
        const int64_t cb = cdiv(q.dv, q.step_cols);
        if (!fits(xcd_grid(q.B * q.Hv * cb, cb), 256)) return PGF_ERR_UNSUPPORTED;
        *out = q;
        return PGF_OK;
    }
    q.chunks_per = cdiv(q.L, kC);
    q.chunk_slots = p->n_seqs ? q.L / kC + p->n_seqs : q.B * q.chunks_per;
    if (q.chunk_slots * q.Hv > kMaxItems / col_blocks || q.nseq * q.Hv > kMaxItems / col_blocks)
        return PGF_ERR_UNSUPPORTED;
    q.seg = p->seg_len > 0 ? p->seg_len : p->seg_len < 0 ? 0 : default_seg(q, p->n_seqs > 0, grads);
    if (q.seg >= q.L) q.seg = 0;
    q.segs_per = q.seg ? cdiv(q.L, q.seg) : 1;
    q.seg_slots = !q.seg ? q.nseq : p->n_seqs ? q.L / q.seg + p->n_seqs : q.B * q.segs_per;
    q.supers_per = cdiv(q.L, kSuper * kC);
    q.super_slots = p->n_seqs ? q.L / (kSuper * kC) + p->n_seqs : q.B * q.supers_per;
    const int64_t vt = cdiv(q.dv, 16), kt = cdiv(q.dk, 16), rep = q.Hv / q.Hk;
    q.share = !grads && q.seg_slots * q.Hv * vt <= kShareTiles ? 2 : 1;
    // A block's four waves take `tiles` column tiles of a head, `waves` a tile.
    auto heads = [&](int64_t tiles, int64_t waves) {
        const int64_t cb = cdiv(tiles * waves, 4);
        return fits(xcd_grid(q.seg_slots * q.Hv * cb, cb * rep), 256);
    };
    if (!fits(cdiv(q.chunk_slots * q.Hk, 4), 256) || !heads(vt, q.share) ||
        (q.seg && (!heads(vt + kt, 1) || !fits(xcd_grid(q.nseq * q.Hv * vt, vt), 4 * q.DK))) ||
        (grads && !fits(q.super_slots * q.Hk, 512)) || (p->n_seqs && p->clear_rest && !fits(cdiv(q.L, 64), 256)))
        return PGF_ERR_UNSUPPORTED;
    const int64_t cell = q.Hv * q.dk * q.dv * 4, cell_tr = q.Hv * (int64_t)q.DK * q.DK * 4;
    q.rec_bytes = kMatBytes * (grads ? 3 : 2) + 256;
    const int64_t ns = q.seg ? q.seg_slots : 0, nc = grads ? q.chunk_slots : 0, nu = grads ? q.super_slots : 0;
    bool ok = section(&q.total, &q.rec, q.chunk_slots, q.Hv * q.rec_bytes);
    ok = ok && section(&q.total, &q.segE, ns, cell) && section(&q.total, &q.tr, ns, cell_tr);
    ok = ok && section(&q.total, &q.S, nu, cell) && section(&q.total, &q.dS, nu, cell);
    ok = ok && section(&q.total, &q.u, nc, q.Hv * kC * q.dv * 4) && section(&q.total, &q.du, nc, q.Hv * kC * q.dv * 4);
    ok = ok && section(&q.total, &q.trT, grads ? ns : 0, cell_tr) && section(&q.total, &q.dseg, grads ? ns : 0, cell);
    ok = ok && section(&q.total, &q.acc, rep > 1 ? nu : 0, q.Hk * 2 * kSuper * kC * q.dk * 4);
    if (!ok) return PGF_ERR_UNSUPPORTED;
    q.total = std::max<size_t>(q.total, 256);
    *out = q;
    return PGF_OK;
}

}  // namespace gdr

namespace qk {

int make_plan(const pgf_qk_params *p, Plan *out, bool grads) {
    if (!p || !out) return PGF_ERR_INVALID_ARG;
    Plan q{};
    q.B = p->batch; q.Hq = p->q_heads; q.Hk = p->k_heads; q.L = p->seqlen; q.d = p->d_head; q.rot = p->rot;
    if (q.B < 1 || q.Hq < 0 || q.Hk < 0 || q.Hq + q.Hk < 1 || q.L < 0 || q.d < 1 || q.rot < 0)
        return PGF_ERR_INVALID_ARG;
    if (p->in_dtype != PGF_F32 && p->in_dtype != PGF_BF16) return PGF_ERR_INVALID_ARG;
    if (p->norm < PGF_NORM_NONE || p->norm > PGF_NORM_RMS) return PGF_ERR_INVALID_ARG;
    if (!(p->eps >= 0.0f)) return PGF_ERR_INVALID_ARG;
    if (q.rot > q.d || (q.rot && !p->inv_freq)) return PGF_ERR_INVALID_ARG;
    if (q.rot && p->positions && p->pos_bits != 32 && p->pos_bits != 64) return PGF_ERR_INVALID_ARG;
    if (p->pos_stride < 0 || p->pos_stride > kMaxStride) return PGF_ERR_INVALID_ARG;
    if (q.d % 8 || q.d > 512 || q.rot % 16) return PGF_ERR_UNSUPPORTED;
    if (q.B > kMaxBatch || q.Hq > kMaxHeads || q.Hk > kMaxHeads || q.L > kMaxLen) return PGF_ERR_UNSUPPORTED;
    const int64_t unit = p->in_dtype == PGF_BF16 ? 8 : 4;
    const struct { const int64_t (&s)[3]; bool out; int64_t heads; } arrays[] = {
        {p->q_strides, false, q.Hq}, {p->k_strides, false, q.Hk}, {p->q_out_strides, true, q.Hq},
        {p->k_out_strides, true, q.Hk}, {p->dq_strides, false, q.Hq}, {p->dk_strides, false, q.Hk}};
    for (const auto &a : arrays)
        if (!strides_ok(a.s, unit, a.out, q.B, a.heads, q.L, q.d)) return PGF_ERR_INVALID_ARG;
    if ((double)q.B * (double)(q.Hq + q.Hk) * (double)q.L * (double)q.d > 4e18) return PGF_ERR_UNSUPPORTED;
    if ((double)q.B * (double)q.L > (double)kMaxItems) return PGF_ERR_UNSUPPORTED;
    q.G = 1;
    while (q.G * 8 < q.d) q.G *= 2;
    // Steps per block: one while that leaves CUs without a few blocks, then as
    // many as keep those (a block's start, with its angles, costs as much as a
    // few vectors a lane: 16384 steps of 32 heads, two steps a block 112 us,
    // eight 72).
    const int64_t rows = q.B * q.L;
    q.tb = 1;
    while (q.tb < kTurn && rows / (2 * q.tb) >= 1024) q.tb *= 2;
    // Blocks take further steps in turns where a launch would have too many.
    q.blocks = std::min<int64_t>(cdiv(rows, q.tb), int64_t(1) << 23);
    // Blocks of the gradient kernel: enough to fill the GPU several times; each
    // leaves one partial sum of the weights' gradients.
    q.grad_blocks = std::min<int64_t>(std::max<int64_t>(1, cdiv(rows, q.tb)), 1024);
    q.total = grads && (p->w_q || p->w_k) ? (size_t)q.grad_blocks * 2 * q.d * sizeof(float) : 0;
    *out = q;
    return PGF_OK;
}

}  // namespace qk
}  // namespace pgf

extern "C" size_t pgf_gdr_workspace_bytes(const pgf_gdr_params *p) {
    pgf::gdr::Plan q;
    return pgf::gdr::make_plan(p, &q, p && p->grads, false) == PGF_OK ? q.total : 0;
}

extern "C" int pgf_gdr_plan(const pgf_gdr_params *p, int32_t *seg_len) {
    if (!seg_len) return PGF_ERR_INVALID_ARG;
    pgf::gdr::Plan q;
    const int rc = pgf::gdr::make_plan(p, &q, p && p->grads, false);
    if (rc == PGF_OK) *seg_len = (int32_t)q.seg;
    return rc;
}

extern "C" size_t pgf_qk_norm_workspace_bytes(const pgf_qk_params *p) {
    pgf::qk::Plan q;
    return pgf::qk::make_plan(p, &q, true) == PGF_OK ? q.total : 0;
}
