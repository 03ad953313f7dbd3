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

// Work item of a block, items in runs of `run` that read the same keys (the
// column blocks of the value heads of one key head): a run's blocks are on one
// of the 8 XCDs and share its L2, consecutive runs on different ones, so that a
// long sequence's heads spread over the GPU.  The hardware deals blocks to the
// XCDs in turn.  Items from n on (the grid is padded) are not there.
__device__ __forceinline__ uint32_t xcd_item(uint32_t b, uint32_t run) {
    const uint32_t x = b % 8, i = b / 8;
    return (i / run * 8 + x) * run + i % run;
}

typedef uint32_t uintx2 __attribute__((ext_vector_type(2)));
typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));

// A value that is the same in all lanes, held as such.
__device__ __forceinline__ int64_t uni(int64_t x) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
    return (int64_t)((uint64_t)hi << 32 | lo);
}

// Rows of one head from some step on, read and written through a buffer
// descriptor: what lies behind the last live row reads as zero and is not
// written, without a branch or a comparison, as long as rows lie at least their
// width apart (an output's do).  Of an input whose step stride is less, the rows
// behind the last live one read as what lies there of that row.  A lane whose
// element is not there gives the offset kNone.  The byte offset of row t is
// t * st; st is below 2^24 (checked on the host), a chunk below 2^30.
constexpr uint32_t kNone = 0x80000000u;
struct Buf {
    __amdgpu_buffer_rsrc_t r;
    uint32_t st;                     // bytes from row to row
};
// `live` rows of `width` bytes at p, live >= 1
__device__ __forceinline__ Buf make_buf(const void *p, uint32_t st, int live, int width) {
    return Buf{__builtin_amdgcn_make_buffer_rsrc((void *)p, 0, (int)((uint32_t)(live - 1) * st + (uint32_t)width), 0x00020000), st};
}
// Element [b][h][t] of a view, as a base for make_buf (all arguments uniform).
template <typename T>
__device__ __forceinline__ const T *row_ptr(const View &v, int64_t b, int64_t h, int64_t t) {
    return (const T *)uni((int64_t)(uintptr_t)v.at<const T>(b, h, t));
}

// Eight consecutive elements as they lie in memory: converted where they are
// used, since a conversion waits for the load.
template <typename T>
struct Raw8;
template <>
struct Raw8<__bf16> { uintx4 x; };
template <>
struct Raw8<float> { uintx4 x, y; };
template <typename T>
__device__ __forceinline__ Raw8<T> load8(const Buf &b, uint32_t voff, uint32_t soff) {
    Raw8<T> r;
    r.x = __builtin_amdgcn_raw_buffer_load_b128(b.r, voff, soff, 0);
    if constexpr (sizeof(T) == 4) r.y = __builtin_amdgcn_raw_buffer_load_b128(b.r, voff, soff + 16, 0);
    return r;
}
// One element in a register of its own.
template <typename T>
__device__ __forceinline__ uint32_t load1(const Buf &b, uint32_t voff, uint32_t soff) {
    if constexpr (sizeof(T) == 2) return __builtin_amdgcn_raw_buffer_load_b16(b.r, voff, soff, 0);
    else return __builtin_amdgcn_raw_buffer_load_b32(b.r, voff, soff, 0);
}
template <typename T>
__device__ __forceinline__ float raw_f(uint32_t u) { return __builtin_bit_cast(float, sizeof(T) == 2 ? u << 16 : u); }
template <typename T>
__device__ __forceinline__ void store1(const Buf &b, uint32_t voff, uint32_t soff, float x) {
    if constexpr (sizeof(T) == 2)
        __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(unsigned short, (__bf16)x), b.r, voff, soff, 0);
    else __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, x), b.r, voff, soff, 0);
}

// Four consecutive elements.
template <typename T>
struct Raw4;
template <>
struct Raw4<float> {
    floatx4 x;
    __device__ __forceinline__ floatx4 f() const { return x; }
};
template <>
struct Raw4<__bf16> {
    bf16x4 x;
    __device__ __forceinline__ floatx4 f() const { return __builtin_convertvector(x, floatx4); }
};
template <typename T>
__device__ __forceinline__ Raw4<T> load4(const T *p) { return *(const Raw4<T> *)p; }
template <typename T>
__device__ __forceinline__ Raw4<T> zero4() {
    Raw4<T> r;
    r.x = {};
    return r;
}

template <typename T>
__device__ __forceinline__ T *at_off(T *base, uint32_t bytes) { return (T *)((char *)base + (size_t)bytes); }

typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Two f32 as sums of P bf16 numbers each, o[i] the i-th numbers of both: P = 1
// rounds (error 2^-8 relative at most), P = 2 leaves 2^-17, P = 3 nothing (an f32
// has 24 bits, three times eight).  For bf16 inputs P = 1 is exact.  In pairs, as the conversion
// instruction takes them; x - part is the dot product instruction's (-1, 0) . parts
// + x, exact, so that no part is widened to f32 first: 7 instructions for three
// parts of two numbers in place of 11.  An infinite number leaves NaN in its
// neighbour's parts too; neighbours are always summed over together.
template <int P>
__device__ __forceinline__ void split2(floatx2 x, bf16x2 (&o)[P]) {
#pragma unroll
    for (int i = 0; i < P; ++i) {
        o[i] = __builtin_convertvector(x, bf16x2);
        if (i + 1 < P) {
            uint32_t m0 = 0x0000bf80u, m1 = 0xbf800000u;           // (-1, 0), (0, -1)
            asm("" : "+s"(m0), "+s"(m1));      // (as immediate operands they are misread)
            x[0] = __builtin_amdgcn_fdot2_f32_bf16(o[i], __builtin_bit_cast(bf16x2, m0), x[0], false);
            x[1] = __builtin_amdgcn_fdot2_f32_bf16(o[i], __builtin_bit_cast(bf16x2, m1), x[1], false);
        }
    }
}

// Four numbers' parts.
template <int P>
__device__ __forceinline__ void split4(const floatx4 &x, bf16x4 (&o)[P]) {
    bf16x2 a[P], b[P];
    split2<P>(floatx2{x[0], x[1]}, a);
    split2<P>(floatx2{x[2], x[3]}, b);
#pragma unroll
    for (int i = 0; i < P; ++i) o[i] = __builtin_shufflevector(a[i], b[i], 0, 1, 2, 3);
}

template <int P>
struct Frag { bf16x8 p[P]; };

// Eight f32 -> operand; two accumulator tiles one below the other make one
// operand of the products that contract over their 32 rows (see mfma below).
template <int P>
__device__ __forceinline__ Frag<P> to_frag(const floatx4 &lo, const floatx4 &hi) {
    Frag<P> f;
    bf16x4 a[P], b[P];
    split4<P>(lo, a);
    split4<P>(hi, b);
#pragma unroll
    for (int i = 0; i < P; ++i) f.p[i] = __builtin_shufflevector(a[i], b[i], 0, 1, 2, 3, 4, 5, 6, 7);
    return f;
}

// Parts of eight loaded elements (a bf16's only part is itself).
template <int P>
__device__ __forceinline__ Frag<P> raw_frag(const Raw8<__bf16> &r) {
    static_assert(P == 1, "");
    Frag<P> f;
    f.p[0] = __builtin_bit_cast(bf16x8, r.x);
    return f;
}
template <int P>
__device__ __forceinline__ Frag<P> raw_frag(const Raw8<float> &r) {
    return to_frag<P>(__builtin_bit_cast(floatx4, r.x), __builtin_bit_cast(floatx4, r.y));
}

// v_mfma_f32_16x16x32_bf16: lane (q, c) = (l / 16, l % 16) supplies eight
// elements of row c of A and of column c of B, the same eight contraction
// indexes in both (its "slots"), and receives D[4q + r][c].  Which index a slot
// stands for is free as long as A and B agree, and so is the key that a row of
// the state's tiles stands for:
//   keys   tile 2 i + h, row 4 q + j is key 32 i + 8 q + 4 h + j, so slot 4 h + j
//          of quad q is key 8 q + 4 h + j: two tiles are, as they lie, the B
//          operand of products with K's rows in their natural order
//   steps  tile h, row 4 q + j is step 16 h + 4 q + j, slot 4 h + j of quad q: two
//          tiles are the B operand as they lie; T and A are stored in slot
//          order (perm32), K by key is read by the transposing LDS read, four
//          steps at a time
__device__ __forceinline__ floatx4 mfma(const bf16x8 &a, const bf16x8 &b, const floatx4 &c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
// Position of step i of a chunk in slot order.
__device__ __forceinline__ constexpr int perm32(int i) { return (i & 15) / 4 * 8 + (i >> 4) * 4 + (i & 3); }

// Byte offset of 16-byte unit u of a row in LDS.  Rows are not padded; the
// units of a row are permuted by an exclusive or with the row's number so that
// the same unit of 16 rows spreads over all banks.  Rows of DK bf16, and of 32.
template <int DK>
__device__ __forceinline__ constexpr uint32_t unit_off(int row, int u) {
    return (uint32_t)(row * (DK * 2) + ((u ^ (DK == 128 ? row & 15 : DK == 64 ? row >> 1 & 7 : row >> 2 & 3)) << 4));
}

// Rows t0 + 0..3 of four columns each, transposed by the read: lane i of 16
// gives the address of row i / 4's columns 4 (i % 4).. and receives column i of the
// four rows.
__device__ __forceinline__ bf16x4 read_tr(const void *p) {
    typedef short shortx4 __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                          (__attribute__((address_space(3))) shortx4 *)p));
}

// c + A B with A = sum of PA, B = sum of PB numbers; products below the
// smallest kept part of either are left out (3 and 3 parts: 6 products, 2^-24
// relative to the factors; 2 and 2 parts: 3 products, 2^-15).
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

// The same for N row tiles of A, in turn: a product waits for the one before it
// where both add to the same tile.
template <int PA, int PB, int N>
__device__ __forceinline__ void mfma_parts2(const Frag<PA> (&a)[N], const Frag<PB> &b, floatx4 *c) {
    constexpr int M = PA > PB ? PA : PB;
#pragma unroll
    for (int s = M - 1; s >= 0; --s)
#pragma unroll
        for (int i = 0; i < PA; ++i)
            if (s - i >= 0 && s - i < PB) {
#pragma unroll
                for (int n = 0; n < N; ++n) c[n] = mfma(a[n].p[i], b.p[s - i], c[n]);
            }
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

// A chunk's record (k_gdr_prep): TW, TA and for the gradients T^, as their tiles
// (0,0), (1,0), (1,1) of 16 x 16 f32 (1 KB each; what is above them is zero), then
// e^G of the 32 steps.
constexpr uint32_t kTile = 1024, kMat = 3 * kTile;
__host__ __device__ constexpr uint32_t rec_eG(bool grads) { return (grads ? 3 : 2) * kMat; }
__host__ __device__ constexpr uint32_t rec_bytes(bool grads) { return rec_eG(grads) + 256; }
// In LDS they are images [32][32] of bf16, one a part (unit_off<32>, columns in
// slot order).
constexpr uint32_t kImg = 2048;

// Lane (r, q) = (l / 4, l % 4) holds columns 4 q .. of row r of tile t: P parts of
// it into images m[0] ..
template <int P>
__device__ __forceinline__ void put_tile(char (*m)[kImg], int t, const uintx4 &x) {
    const int l = threadIdx.x % 64;
    const uint32_t at = unit_off<32>(l / 4, l % 4) + (t > 0 ? 16 * 64 : 0) + (t > 1 ? 8 : 0);
    bf16x4 o[P];
    split4<P>(__builtin_bit_cast(floatx4, x), o);
#pragma unroll
    for (int p = 0; p < P; ++p) *(bf16x4 *)&m[p][at] = o[p];
}
// Tile (0,1) of N images: zero, once.
template <int N, int NT>
__device__ __forceinline__ void zero_tile(char (*m)[kImg], int tid) {
    const bf16x4 zero = {};
    for (int i = tid; i < N * 64; i += NT) *(bf16x4 *)&m[i / 64][unit_off<32>(i % 64 / 4, i % 4) + 8] = zero;
}

}  // namespace gdr
}  // namespace pgf
