// Host-side planning of the gated delta rule and of the query/key
// preparation: argument checks and workspace layout.  Plain C++ without
// device access.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "../../include/pgf.h"

namespace pgf {
namespace gdr {

constexpr int kC = 32;           // steps per chunk
constexpr int kSuper = 2;        // chunks between saved states of the gradients
// Column tiles of the scan's outputs up to which two waves share one (k_gdr_chain).
constexpr int64_t kShareTiles = 512;
constexpr int64_t kMatBytes = 3 * 1024;  // a chunk's lower triangular matrix: three 16 x 16 tiles of f32

// Blocks for n items in runs of `run` that are dealt to the 8 XCDs (xcd_item).  The
// planner sees to it that a launch has fewer than 2^32 threads.
inline int64_t xcd_grid(int64_t n, int64_t run) {
    const int64_t runs = (n + run - 1) / run;
    return (runs + 7) / 8 * 8 * run;
}

// Workspace sections (bytes, 256-byte aligned).
//   rec   [chunk slots][Hv]                   k_gdr_prep's record of each chunk
//   seg   [segment slots][Hv][dk][dv]         zero-start end state of a segment,
//                                             then (in place) its entry state
//   tr    [segment slots][Hv][DK][DK]         transition of a segment
// gradients:
//   S     [super slots][Hv][dk][dv]           state entering every kSuper chunks
//   dS    [super slots][Hv][dk][dv]           its adjoint leaving them
//   u, du [chunk slots][Hv][32][dv]           E and its adjoint of each chunk
//   trT   [segment slots][Hv][DK][DK]         tr transposed
//   dseg  [segment slots][Hv][dk][dv]         as seg, of the adjoint
//   acc   [super slots][Hk][2][64][dk]        sums of dq and dk over value heads, where
//                                             a key head has several
struct Plan {
    int64_t B, Hk, Hv, L, dk, dv, nseq;
    int DK;                      // d_key padded to the kernels' 64 or 128
    int64_t chunk_slots, chunks_per;     // slots of kC steps, of a dense sequence
    int64_t seg;                 // steps per segment, 0 = sequences are not cut
    int64_t seg_slots, segs_per;
    int64_t super_slots, supers_per;     // slots of kSuper * kC steps
    int share;                   // waves that share a column tile of the scan's outputs
    int step_cols;               // value columns of a block of single steps
    int64_t rec_bytes;           // of one chunk's record
    size_t rec, segE, tr, S, dS, u, du, trT, dseg, acc, total;
};

// Validates sizes, types and strides, not pointers.  step: of pgf_gdr_step.
int make_plan(const pgf_gdr_params *p, Plan *q, bool grads, bool step);

}  // namespace gdr

namespace qk {

constexpr int kTurn = 8;         // steps per block and turn at most

struct Plan {
    int64_t B, Hq, Hk, L, d, rot;
    int G;                       // lanes per head
    int tb;                      // steps per block and turn
    int64_t blocks, grad_blocks; // blocks of the kernel, and of the gradients'
    size_t total;
};
int make_plan(const pgf_qk_params *p, Plan *q, bool grads);

}  // namespace qk

// Strides {0,0,0} stand for dense rows of `width` elements in [.., heads, L, width].
// A single step's row ends with its width, whatever stride its step index has (a
// slice's, or zero): kernels bound rows by the step stride.
void dense_strides(const int64_t (&in)[3], int64_t heads, int64_t L, int64_t width, int64_t (&out)[3]);
// Bytes from the first to behind the last element of such an array (0 if empty).
size_t extent(const int64_t (&s)[3], int64_t B, int64_t heads, int64_t L, int64_t width, size_t elem);
bool overlaps(const void *a, size_t na, const void *b, size_t nb);

// An array of rows as it lies in memory (strides in elements, {0,0,0} dense).
struct Arr {
    const void *p;
    const int64_t (&s)[3];
    int64_t B, H, L, width;
    size_t elem;
    size_t bytes() const { return extent(s, B, H, L, width, elem); }
};
// Whether two such arrays may share memory.  Arrays whose rows interleave (parts of
// one fused array's rows, or of its heads' rows) do not.
bool overlaps(const Arr &a, const Arr &b);

}  // namespace pgf
