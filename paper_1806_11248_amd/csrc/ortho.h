// What the kernels of orthogonalised updates and their entry points share.
#pragma once

#include "gbt_internal.h"

constexpr int kOrthoTile = 128;         // rows and columns that a workgroup computes of a product
constexpr int kOrthoPiece = 1 << 14;    // elements whose squares a workgroup adds up

// One update in the device's list.  The shorter side is `p`, the longer one `w`: X is p x w, G or its transpose.  Both are padded with zeros to whole
// tiles in the workspace.
struct OrthoMatrix {
    const void *src;
    void *dst;
    int64_t cols;                       // of G
    int32_t p, w, pp, ww;               // ww, pp: padded
    int32_t tall, dtype;                // tall: X is G's transpose
    float scale;
    int32_t pieces;                     // of its elements
    int64_t piece_begin;                // of the group's pieces
    int64_t x[2], xt[2], a, b;          // bytes into the workspace: X and its transpose, twice, and the two p x p matrices; each a plane of high parts, then one of low parts
    int64_t fill_begin, sym_begin, full_begin;   // of the group's tiles: of X, of symmetric products' upper halves, of X
};

struct OrthoArgs {
    const OrthoMatrix *list;            // of the group
    int count;
    char *workspace;
    double *squares;                    // [pieces of the group]
    float a, b, c;
    int from, last;                     // which of the two X is read; whether this is the last step
};

hipError_t gbt_launch_ortho_begin(hipStream_t stream, const OrthoArgs &a, int64_t pieces, int64_t fill_tiles);
hipError_t gbt_launch_ortho_step(hipStream_t stream, const OrthoArgs &a, int64_t sym_tiles, int64_t full_tiles);
