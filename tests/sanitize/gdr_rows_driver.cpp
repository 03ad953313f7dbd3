// The rows of arrays as the kernels of the gated delta rule take them (host
// planning alone, no device).  The chains write a chunk's 32 rows through a
// buffer that ends with the last live row, at t * (step stride) for row t: for
// every output whose strides the planner accepts, the rows behind the last
// live one lie behind that end.
//   one     arrays of one step, whatever stride their step index has
//   apart   arrays of any length; and no two rows of an accepted output share an
//           element
//   parts   parts of one array's rows do not count as overlapping, in any order of
//           batch, head and step, and arrays that share an element do
#include <stdio.h>
#include <string.h>

#include <random>
#include <set>

#include "../../paper_2512_23068_amd/csrc/pgf_gdr_plan.h"

// q, k and v (or their gradients) as parts of one array's rows.
static int parts() {
    std::mt19937_64 rng(9);
    auto pick = [&](std::initializer_list<int64_t> v) { return *(v.begin() + rng() % v.size()); };
    static char mem[1 << 20];
    long apart = 0, shared = 0, failures = 0;
    for (int i = 0; i < 20000; ++i) {
        const int64_t n[3] = {pick({1, 2, 3}), pick({1, 2, 4}), pick({1, 2, 5})};
        const int64_t w[2] = {pick({8, 16, 24}), pick({8, 16})}, gap = pick({0, 0, 8});
        const bool inner = rng() % 2;              // each part's heads side by side, or heads of all parts
        int order[3] = {0, 1, 2};
        for (int k = 2; k > 0; --k) std::swap(order[k], order[rng() % (k + 1)]);
        int64_t s[2][3], at, H[2] = {n[1], inner ? pick({1, 2, 4}) : n[1]};
        if (inner) {                               // [.., step (or batch), heads of the first, heads of the second]
            at = H[0] * w[0] + gap;
            int64_t step = at + H[1] * w[1] + pick({0, 8});
            for (int k = 0; k < 2; ++k) s[k][1] = w[k];
            for (int k : order)
                if (k != 1) {
                    s[0][k] = s[1][k] = step;
                    step *= n[k];
                }
        } else {                                   // rows [first, second] of any order
            at = w[0] + gap;
            int64_t step = at + w[1] + pick({0, 8});
            for (int k : order) {
                s[0][k] = s[1][k] = step;
                step *= n[k];
            }
        }
        const int64_t move = rng() % 2 ? 0 : pick({-8, 8, 16});      // (the second part out of its place)
        if (at + move < 0) continue;
        const pgf::Arr a{mem, s[0], n[0], H[0], n[2], w[0], 2}, b{mem + 2 * (at + move), s[1], n[0], H[1], n[2], w[1], 2};
        std::set<int64_t> first;
        bool hit = false;
        for (int k = 0; k < 2; ++k)
            for (int64_t x = 0; x < n[0]; ++x)
                for (int64_t h = 0; h < H[k]; ++h)
                    for (int64_t t = 0; t < n[2]; ++t)
                        for (int64_t e = 0; e < w[k]; ++e) {
                            const int64_t y = x * s[k][0] + h * s[k][1] + t * s[k][2] + e + (k ? at + move : 0);
                            if (!k) first.insert(y);
                            else hit |= first.count(y) > 0;
                        }
        (hit ? shared : apart) += 1;
        const bool found = pgf::overlaps(a, b) || pgf::overlaps(b, a);
        if (hit ? !(pgf::overlaps(a, b) && pgf::overlaps(b, a)) : !move && found) ++failures;
    }
    printf("%ld pairs apart, %ld share elements, %ld failures\n", apart, shared, failures);
    return apart > 1000 && shared > 1000 ? 0 : 1;
}

int main(int argc, char **argv) {
    if (argc > 1 && !strcmp(argv[1], "parts")) return parts();
    const bool one = argc > 1 && !strcmp(argv[1], "one");
    std::mt19937_64 rng(7);
    auto pick = [&](std::initializer_list<int64_t> v) { return *(v.begin() + rng() % v.size()); };
    long accepted = 0, failures = 0;
    for (int i = 0; i < 100000; ++i) {
        pgf_gdr_params p;
        memset(&p, 0, sizeof(p));
        p.batch = pick({1, 2, 3});
        p.key_heads = pick({1, 2});
        p.value_heads = p.key_heads * pick({1, 2});
        p.seqlen = one ? 1 : pick({1, 2, 31, 33, 70});
        p.d_key = pick({8, 64, 128});
        p.d_value = pick({8, 40, 64, 200});
        p.in_dtype = (int)pick({0, 1});
        p.scale = 1.0f;
        const int64_t e = p.in_dtype ? 2 : 4;
        const bool grads = rng() % 2;
        struct { int64_t (&s)[3]; int64_t heads, width; } outs[] = {
            {p.o_strides, p.value_heads, p.d_value}, {p.dq_strides, p.key_heads, p.d_key},
            {p.dk_strides, p.key_heads, p.d_key}, {p.dv_strides, p.value_heads, p.d_value}};
        for (int k = 0; k < 4; ++k) {
            if ((k == 0) == grads || rng() % 2) continue;          // (not an output of this call, or dense)
            auto &o = outs[k];
            const int64_t w = o.width, n = o.heads;
            o.s[2] = pick({0, 8, w, n * w, n * w + 64});
            o.s[1] = pick({w, w * p.seqlen, 8, n > 1 ? w : 0});
            o.s[0] = pick({n * w * p.seqlen, (n * w + 64) * p.seqlen, p.batch > 1 ? n * w : 0});
        }
        pgf::gdr::Plan q;
        if (pgf::gdr::make_plan(&p, &q, grads, false) != PGF_OK) continue;
        ++accepted;
        for (int k = 0; k < 4; ++k) {
            if ((k == 0) == grads) continue;
            const auto &o = outs[k];
            int64_t d[3];
            pgf::dense_strides(o.s, o.heads, q.L, o.width, d);
            const int64_t live = (q.L - 1) % 32 + 1, end = ((live - 1) * d[2] + o.width) * e;
            for (int64_t t = live; t < 32; ++t)
                if (t * d[2] * e < end) {
                    ++failures;
                    break;
                }
        }
    }
    // rows of outputs against their elements themselves; rows in whatever order,
    // as long as the longer strides step over what the shorter ones span, are taken
    long nested = 0;
    for (int i = 0; i < 20000 && !one; ++i) {
        pgf_gdr_params p;
        memset(&p, 0, sizeof(p));
        p.batch = pick({1, 2, 3});
        p.key_heads = p.value_heads = pick({1, 2, 3});
        p.seqlen = pick({1, 2, 5});
        p.d_key = p.d_value = 8;
        p.in_dtype = 1;
        const int64_t n[3] = {p.batch, p.value_heads, p.seqlen};
        int order[3] = {0, 1, 2};
        for (int k = 2; k > 0; --k) std::swap(order[k], order[rng() % (k + 1)]);
        int64_t span = 8;
        for (int k : order) {
            p.o_strides[k] = span + pick({0, 0, 8, 16});
            span = (n[k] - 1) * p.o_strides[k] + span;
            span = (span + 7) / 8 * 8;
        }
        bool clash = false;
        const bool change = rng() % 2;
        if (change) p.o_strides[rng() % 3] = pick({8, 16, 24, 32, 48});
        std::set<int64_t> seen;
        for (int64_t b = 0; b < n[0]; ++b)
            for (int64_t h = 0; h < n[1]; ++h)
                for (int64_t t = 0; t < n[2]; ++t)
                    for (int64_t x = 0; x < 8; ++x)
                        clash |= !seen.insert(b * p.o_strides[0] + h * p.o_strides[1] + t * p.o_strides[2] + x).second;
        pgf::gdr::Plan q;
        const bool ok = pgf::gdr::make_plan(&p, &q, false, false) == PGF_OK;
        if ((ok && clash) || (!ok && !change)) ++failures;
        nested += ok;
    }
    if (!one && nested < 1000) ++failures;
    printf("%ld plans accepted, %ld failures\n", accepted, failures);
    return accepted > 1000 ? 0 : 1;
}
