// Shared by the kernels of the gated delta rule (pgf_gdr.hip, its gradients in
// pgf_gdr_grads.hip) and of the query/key preparation (pgf_qk.hip): strided
// views, loads of f32 and bf16 rows, and products on the bf16 matrix cores
// whose f32 operands enter as sums of bf16 numbers.
#pragma once

#include <hip/hip_runtime.h>

#include <stdint.h>

#include "pgf_gdr_plan.h"

namespace pgf {
namespace gdr {

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef unsigned short ushortx4 __attribute__((ext_vector_type(4)));

// An array [batch][head][step][dense index] with strides in elements.
struct View {
    const void *p;
    int64_t sb, sh, st;
    template <typename T>
    __device__ __forceinline__ T *at(int64_t b, int64_t h, int64_t t) const {
        return (T *)p + (b * sb + h * sh + t * st);
    }
};

// Block barrier that orders LDS only: global loads and stores stay in flight.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// LDS written and read again by one wave: its accesses execute in order, the
// compiler must not move them across this.
__device__ __forceinline__ void wave_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Block number -> work item so that neighbours in the work order (column
// blocks of one head, which read the same keys) run on one of the 8 XCDs and
// share its L2; the hardware deals blocks to the XCDs in turn.
__device__ __forceinline__ uint32_t xcd_order(uint32_t b, uint32_t n) {
    const uint32_t per = n / 8, rem = n % 8, x = b % 8;
    return x * per + (x < rem ? x : rem) + b / 8;
}

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__bf16 x) { return (float)x; }

template <typename T>
struct Vec4 { T v[4]; };          // 4 consecutive elements, as loaded

__device__ __forceinline__ Vec4<float> load4(const float *p) {
    const floatx4 x = *(const floatx4 *)p;
    return {{x[0], x[1], x[2], x[3]}};
}
__device__ __forceinline__ Vec4<__bf16> load4(const __bf16 *p) {
    const bf16x4 x = *(const bf16x4 *)p;
    return {{x[0], x[1], x[2], x[3]}};
}
template <typename T>
__device__ __forceinline__ Vec4<T> zero4() {
    return {{(T)0.0f, (T)0.0f, (T)0.0f, (T)0.0f}};
}

// bf16 numbers whose sum is x: P = 1 rounds (error 2^-9 relative), P = 2 leaves
// 2^-18, P = 3 2^-27 (below an f32's own rounding).  For a bf16 input P = 1 is
// exact.
template <int P>
__device__ __forceinline__ void split(float x, __bf16 (&o)[P]) {
    o[0] = (__bf16)x;
    if constexpr (P > 1) {
        const float r = x - (float)o[0];
        o[1] = (__bf16)r;
        if constexpr (P > 2) o[2] = (__bf16)(r - (float)o[1]);
    }
}

template <int P>
struct Frag { bf16x8 p[P]; };

// Eight f32 -> operand; two accumulator tiles one below the other make one
// operand of the products that contract over their 32 rows (see mfma below).
template <int P>
__device__ __forceinline__ Frag<P> to_frag(const floatx4 &lo, const floatx4 &hi) {
    Frag<P> f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        __bf16 a[P], b[P];
        split<P>(lo[j], a);
        split<P>(hi[j], b);
#pragma unroll
        for (int i = 0; i < P; ++i) {
            f.p[i][j] = a[i];
            f.p[i][4 + j] = b[i];
        }
    }
    return f;
}

// v_mfma_f32_16x16x32_bf16: lane (q, c) = (l / 16, l % 16) supplies eight
// elements of row c of A and of column c of B, the same eight contraction
// indexes in both, and receives D[4q + r][c].  Which index a slot stands for
// is free as long as A and B agree.  Here slot (q, j) of a block of 32 is
// index 4q + j (j < 4) or 16 + 4q + j - 4, so that two accumulator tiles are
// a B operand as they lie; in memory a row is stored in slot order
// (perm32 below), so that an A operand is one 16-byte read.
__device__ __forceinline__ floatx4 mfma(const bf16x8 &a, const bf16x8 &b, const floatx4 &c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Position of index i of a block of 32 in slot order.
__device__ __forceinline__ constexpr int perm32(int i) { return (i & 15) / 4 * 8 + (i >> 4) * 4 + (i & 3); }

// c + A B with A = sum of PA, B = sum of PB numbers; products below the
// smallest kept part of either are left out (3 and 3 parts: 6 products).
template <int PA, int PB>
__device__ __forceinline__ floatx4 mfma_parts(const Frag<PA> &a, const Frag<PB> &b, floatx4 c) {
    constexpr int N = PA > PB ? PA : PB;
#pragma unroll
    for (int s = N - 1; s >= 0; --s)
#pragma unroll
        for (int i = 0; i < PA; ++i)
            if (s - i >= 0 && s - i < PB) c = mfma(a.p[i], b.p[s - i], c);
    return c;
}

// The sequence that slot number i of `unit` steps belongs to, and its rows.
// Dense batches have `per` slots a sequence; packed ones number the slots of
// sequence n from cu[n] / unit + n on (ceil(len / unit) of them, which never
// reaches the next sequence's first).
struct Rows {
    int64_t b, n;        // batch entry, sequence
    int64_t lo;          // first row of the sequence
    int64_t len;         // its steps
    int64_t unit0;       // first step of the slot, within the sequence (may lie behind its end)
};
struct Seqs {
    const int32_t *cu;
    int64_t n, L;
    __device__ __forceinline__ int64_t bound(int64_t i) const {
        const int64_t x = cu[i];
        return x < 0 ? 0 : (x > L ? L : x);
    }
    __device__ __forceinline__ int64_t slot0(int64_t s, int64_t unit, int64_t per) const {
        return cu ? bound(s) / unit + s : s * per;
    }
    __device__ __forceinline__ Rows of(int64_t i, int64_t unit, int64_t per) const {
        Rows r;
        if (!cu) {
            r.b = r.n = i / per;
            r.lo = 0;
            r.len = L;
            r.unit0 = (i - r.n * per) * unit;
            return r;
        }
        int64_t a = 0, e = n - 1;      // last n with slot0(n) <= i
        while (a < e) {
            const int64_t m = (a + e + 1) / 2;
            if (bound(m) / unit + m <= i) a = m; else e = m - 1;
        }
        r.b = 0;
        r.n = a;
        r.lo = bound(a);
        const int64_t hi = bound(a + 1);
        r.len = hi > r.lo ? hi - r.lo : 0;
        r.unit0 = (i - (r.lo / unit + a)) * unit;
        if (r.unit0 < 0) r.unit0 = r.len;      // (cu not ascending)
        return r;
    }
};

// Floats of a chunk's record (k_gdr_prep): T and A as three 16 x 16 blocks
// each ((0,0), (1,0), (1,1), row-major), then e^G, e^{G_end - G} and beta of
// its 32 steps.
constexpr int kRecT = 0, kRecA = 768, kRecRow = 1536, kRec = 1632;

}  // namespace gdr
}  // namespace pgf
