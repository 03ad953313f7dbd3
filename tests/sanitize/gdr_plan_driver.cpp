// Host planning of the gated delta rule and the query/key preparation
// (make_plan, extent, overlaps: plain C++, no device) for a build with
// AddressSanitizer and UndefinedBehaviorSanitizer: random sizes and strides up
// to and beyond every limit are refused or give sections in order within the
// workspace, and overlaps agrees with a count of shared bytes.
#include <stdio.h>
#include <string.h>

#include <random>
#include <set>

#include "../../paper_2512_23068_amd/csrc/pgf_gdr_plan.h"

int main() {
    std::mt19937_64 rng(1);
    auto pick = [&](std::initializer_list<int64_t> v) { return *(v.begin() + rng() % v.size()); };
    long failures = 0, accepted = 0, shared = 0;
    for (int i = 0; i < 200000; ++i) {
        pgf_gdr_params p;
        memset(&p, 0, sizeof(p));
        p.batch = pick({1, 2, 7, 1000, 1 << 24, (int64_t)1 << 62, 0, -3});
        p.key_heads = pick({1, 2, 16, 1 << 16, (int64_t)1 << 40});
        p.value_heads = p.key_heads * pick({1, 2, 4});
        p.seqlen = pick({0, 1, 31, 64, 1000, 131072, (int64_t)1 << 32, (int64_t)1 << 33, -1});
        p.d_key = pick({8, 16, 64, 72, 128, 136, 12});
        p.d_value = pick({8, 64, 200, 4096, 4104});
        p.n_seqs = pick({0, 0, 1, 9, 100000});
        p.in_dtype = (int)pick({0, 1, 1, 2});
        p.seg_len = (int)pick({0, 0, -1, 64, 4096, 1 << 30, 33});
        int64_t(*st[9])[3] = {&p.q_strides, &p.k_strides, &p.v_strides, &p.g_strides, &p.beta_strides, &p.o_strides,
                              &p.dq_strides, &p.dk_strides, &p.dv_strides};
        if (i % 3 == 0)
            for (auto *s : st)
                for (auto &x : *s) x = pick({0, 8, 64, 4096, (int64_t)1 << 22, (int64_t)1 << 44, ((int64_t)1 << 44) + 8, -8});
        for (int g = 0; g < 3; ++g) {
            pgf::gdr::Plan q;
            const int rc = pgf::gdr::make_plan(&p, &q, g == 1, g == 2);
            if (rc > 0 || rc < -2) ++failures;
            if (rc != PGF_OK) continue;
            ++accepted;
            (void)pgf::extent(p.q_strides, q.B, q.Hk, q.L, q.dk, 4);
            (void)pgf::extent(p.o_strides, q.B, q.Hv, q.L, q.dv, 4);
            if (g == 2) continue;
            const size_t at[] = {q.rec, q.segE, q.tr, q.S, q.dS, q.u, q.du, q.trT, q.dseg, q.acc, q.total};
            for (int k = 0; k + 1 < 11; ++k)
                if (at[k] > at[k + 1] || at[k] % 256) ++failures;
            if (q.seg % 64 || (q.seg && q.seg >= q.L)) ++failures;
        }
        pgf_qk_params k;
        memset(&k, 0, sizeof(k));
        k.batch = p.batch; k.q_heads = p.key_heads; k.k_heads = pick({0, 1, 16}); k.seqlen = p.seqlen;
        k.d_head = pick({8, 72, 128, 512, 520, 20}); k.rot = pick({0, 16, 64, 512, 24}); k.in_dtype = p.in_dtype;
        k.norm = (int)pick({0, 1, 2, 3}); k.inv_freq = (const float *)16;
        memcpy(k.q_strides, p.q_strides, sizeof(k.q_strides));
        pgf::qk::Plan q;
        const int rc = pgf::qk::make_plan(&k, &q, true);
        if (rc > 0 || rc < -2 || (rc == PGF_OK && (q.G * 8 < q.d || q.G > 64))) ++failures;
    }
    // overlaps against the bytes themselves: never "apart" where bytes are shared
    static char mem[1 << 16];
    for (int i = 0; i < 20000; ++i) {
        const int64_t B = pick({1, 2, 3}), L = pick({1, 2, 5});
        int64_t s[2][3], H[2], w[2];
        const int64_t st = pick({8, 16, 24, 48}), sb = pick({48, 96, 240, 480});
        for (int k = 0; k < 2; ++k) {
            H[k] = pick({1, 2});
            w[k] = pick({8, 16});
            s[k][0] = pick({sb, sb, 240});
            s[k][1] = pick({w[k], w[k], 100});
            s[k][2] = pick({st, st, 16});
        }
        const int64_t at = (int64_t)(rng() % 600);
        const pgf::Arr a{mem, s[0], B, H[0], L, w[0], 2}, b{mem + 2 * at, s[1], B, H[1], L, w[1], 2};
        std::set<int64_t> bytes;
        bool hit = false;
        for (int k = 0; k < 2; ++k)
            for (int64_t bb = 0; bb < B; ++bb)
                for (int64_t h = 0; h < H[k]; ++h)
                    for (int64_t t = 0; t < L; ++t)
                        for (int64_t e = 0; e < w[k]; ++e) {
                            const int64_t x = bb * s[k][0] + h * s[k][1] + t * s[k][2] + e + (k ? at : 0);
                            if (!k) bytes.insert(x);
                            else hit |= bytes.count(x) > 0;
                        }
        shared += hit;
        if (hit && !pgf::overlaps(a, b)) ++failures;
    }
    printf("%ld plans accepted, %ld pairs share bytes, %ld failures\n", accepted, shared, failures);
    return accepted > 1000 && shared > 1000 ? 0 : 1;
}
