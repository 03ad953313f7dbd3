// Launches of the gated delta rule and the query/key preparation (host planning
// alone, no device): a launch of 2^32 threads or more runs only the low 32 bits of
// their number, so every plan that is accepted launches fewer, and steps that
// launch fewer are accepted.
#include <stdio.h>
#include <string.h>

#include <random>

#include "../../paper_2512_23068_amd/csrc/pgf_gdr_plan.h"

using i64 = int64_t;
static i64 up(i64 a, i64 b) { return (a + b - 1) / b; }
static bool fits(i64 blocks, i64 threads) { return (double)blocks * (double)threads < 4294967296.0; }
// n items in runs, runs dealt to 8 parts of the GPU
static i64 dealt(i64 n, i64 run) { return up(up(n, run), 8) * 8 * run; }

int main() {
    std::mt19937_64 rng(3);
    auto pick = [&](std::initializer_list<i64> v) { return *(v.begin() + rng() % v.size()); };
    long accepted = 0, beyond = 0, failures = 0;
    for (int i = 0; i < 400000; ++i) {
        pgf_gdr_params p;
        memset(&p, 0, sizeof(p));
        p.batch = (i64)1 << rng() % 22;
        p.batch += pick({-1, 0, 0, 1});
        p.key_heads = (i64)1 << rng() % 8;
        p.value_heads = p.key_heads * pick({1, 1, 2, 16});
        p.seqlen = pick({1, 2, 33, 65, 1000, 131072, ((i64)1 << 30) - 64, (i64)1 << 31});
        p.d_key = pick({8, 64, 72, 128});
        p.d_value = pick({8, 64, 136, 512});
        p.seg_len = (int)pick({0, -1, 64});
        p.clear_rest = (int)pick({0, 1});
        if (rng() % 3 == 0) {
            p.n_seqs = p.batch;
            p.batch = 1;
        }
        if (p.batch < 1) continue;
        for (int g = 0; g < 3; ++g) {
            if (g == 2 && p.n_seqs) continue;
            pgf::gdr::Plan q;
            const int rc = pgf::gdr::make_plan(&p, &q, g == 1, g == 2);
            const i64 vt = up(p.d_value, 16), kt = up(p.d_key, 16), rep = p.value_heads / p.key_heads;
            const i64 n = p.n_seqs ? p.n_seqs : p.batch;
            bool ok = true;
            if (g == 2) {
                const bool wide = p.seqlen > 2 && p.batch * p.value_heads * up(p.d_value, 128) >= 256;
                const i64 cb = up(p.d_value, wide ? 128 : 32);
                ok = fits(dealt(p.batch * p.value_heads * cb, cb), 256);
            } else if (rc == PGF_OK) {
                ok = fits(up(q.chunk_slots * q.Hk, 4), 256);
                if (q.seg) {
                    ok = ok && fits(dealt(q.seg_slots * q.Hv * up(vt + kt, 4), up(vt + kt, 4) * rep), 256);
                    ok = ok && fits(dealt(n * q.Hv * vt, vt), 4 * q.DK);
                }
                const i64 cb = g == 0 && q.seg_slots * q.Hv * vt <= 512 ? up(vt, 2) : up(vt, 4);
                ok = ok && fits(dealt(q.seg_slots * q.Hv * cb, cb * rep), 256);
                if (g == 1) ok = ok && fits(q.super_slots * q.Hk, 512);
                if (p.n_seqs && p.clear_rest) ok = ok && fits(up(p.seqlen, 64), 256);
            }
            accepted += rc == PGF_OK;
            beyond += rc == PGF_ERR_UNSUPPORTED;
            if (rc == PGF_OK && !ok) ++failures;
            // (far lengths pass 2^62 elements)
            if (g == 2 && ok && rc != PGF_OK && p.seqlen <= 131072) ++failures;
        }
    }
    for (int i = 0; i < 100000; ++i) {
        pgf_qk_params p;
        memset(&p, 0, sizeof(p));
        p.batch = (i64)1 << rng() % 25;
        p.q_heads = 1;
        p.seqlen = ((i64)1 << rng() % 31) + (i64)(rng() % 3);
        p.d_head = 8;
        pgf::qk::Plan q;
        if (pgf::qk::make_plan(&p, &q, false) != PGF_OK) continue;
        if (!fits(q.blocks, 256) || !fits(q.grad_blocks, 256) || q.blocks < 1 || q.grad_blocks < 1) ++failures;
    }
    printf("%ld plans accepted, %ld refused, %ld failures\n", accepted, beyond, failures);
    return accepted > 1000 && beyond > 1000 ? 0 : 1;
}
