// xent_mma.cuh -- host/device interface of the tensor-core cross entropy.
#pragma once
#include <cuda.h>

#include "xent.cuh"

namespace fibattn {
namespace xent {

constexpr int kClusters = 76;                      // CTA pairs of a GB300 (152 SMs)

// One product of the backward: rows x (tiles of) columns, depth in chunks of 64;
// `siblings` clusters at a time share the column tiles, each has `tiles` tiles.
struct Product {
    int rows, col_tiles, chunks, tiles, siblings;
};

struct Args {
    Problem p;
    // forward and gradient: tiles of 256 x 256, depth in chunks of 64.  A unit
    // of the forward is unit_tiles tiles of one row of tiles.
    int chunks, row_tiles, col_tiles, unit_tiles, units;
    FwdParts parts;
    const float* lse;
    const float* dloss;
    int v0, cols;                                  // the piece of the vocabulary
    Product prob[2];                               // products: dx, dw
    int first_dw, snap[2];                         // the first cluster of dw's
    int tile_cols, out_cols;                       // columns of a tile, of the results (D)
    float* partials;                               // sums over a part of a tile's depth
    float* scale;                                  // g is divided by it, the products multiplied
    const float* maxima;                           // of |dloss|, over parts of the rows (n_maxima may be 0)
    int n_maxima;
    int row_box;                                   // rows of the boxes that x is loaded in
    float* dx_acc;                                 // dx over the earlier pieces, fp32
    bool dx_add, dx_done;                          // there are earlier pieces; this is the last one
    void* dx;
    void* dw;
    bool out_f32;
    // operands of several planes: product i takes planes (combo_a >> 4 i) & 15 and (combo_b >> 4 i) & 15
    int combos;
    unsigned combo_a, combo_b;
};

struct Maps {
    CUtensorMap m[4];
};

// Where a call goes: rows as vectors, few rows, or tiles on the fifth-generation cores.
enum class Way { kStream, kFewRows, kTiles };

struct FwdPlan {
    Way way;
    bool pack, wide;                               // wide: logits of several planes, or in short runs
    int planes, depth;                             // of packed operands: planes, row length
    int unit_tiles, segments;                      // segments: entries of a row in FwdParts
    size_t x, w, m, l, target, total;              // workspace offsets
};
FwdPlan plan_forward(int N, int D, int V, bool bf16);
cudaError_t run_forward(const Problem& p, const FwdPlan& plan, char* ws, bool bf16, float* loss, float* lse, cudaStream_t st);

struct BwdPlan {
    Way way;
    bool pack, wide;                               // wide: products of several planes
    int planes, depth, g_planes;
    int blocks;                                    // blocks of 256 columns of a products' tile
    int ranges;                                    // parts of dx (not for tiles)
    int cols, ldg;                                 // columns of a piece; row length of g
    size_t x, w, g, dx_acc, partials, scale, total;
    int maxima;                                    // blocks that look for the largest |dloss|; 0: not apart
};
BwdPlan plan_backward(int N, int D, int V, bool bf16);
cudaError_t run_backward(const Problem& p, const BwdPlan& plan, char* ws, bool bf16, const float* lse, const float* dloss,
                         void* dx, void* dw, cudaStream_t st);

}  // namespace xent
}  // namespace fibattn
