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
    int32_t p, w, pp, ww;               // pp, ww: padded
    int32_t tall, dtype;                // tall: X is G's transpose
    float scale;
    int32_t pieces;                     // of its elements
    int64_t piece_begin;                // of the group's pieces
    int64_t x, xt[2];                   // bytes into the workspace: X, its transpose (and the next one)
    int64_t gram, factor[2], between, total;   // p x p: A, the factors F of a round's one or two steps, F A between them, and the product of both
    int64_t fill_begin;                 // of the group's workgroups that lay X out
};
// What a workgroup of a product computes: tile (i, j) of one matrix of the group; matrix < 0: nothing.
struct OrthoTile {
    int32_t matrix;
    int16_t i, j;
};

// What is held in two float16 parts is held times a power of two, of which the products' results and the bounds of what comes of them lie up to 2^15, half of
// float16's largest number: a low part stays a normal number, and 22 bits are held, of elements down to 2^-17 of the bound; smaller ones are off by 2^-40 of it.
constexpr float kScaleUp = 32768.0f, kScaleDown = 1.0f / 32768.0f;
struct OrthoScales {
    float x[33];                        // of X before each step and after the last
    float factor[32];                   // of each step's factor; a product of factors is held times the product of their scales, a kScaleUp less for each
    float gram(int s) const { return x[s] * x[s] * kScaleDown; }   // of A; F A is held times that of X before and after the step
    float after(int s) const { return x[s + 1] / (x[s] * factor[s]); }   // from the operands' scales to F A's, and from its and F's to the next A's
    // from the scales of X and of the product of the factors of steps s to e to that of X behind them, or to none behind the last
    float apply(int s, int e, int steps) const {
        float up = (e < steps ? x[e] : 1.0f) / x[s];
        for (int t = s; t < e; ++t) up /= t == s ? factor[t] : factor[t] * kScaleDown;
        return up;
    }
};
// The same as one workgroup takes them, with nothing left to divide.
struct OrthoSmallScales {
    struct Step {
        float less[4];                  // of A A, the product of two factors, F A and F A F
        float gram, factor, apply, none;   // factor: from A's scale to the factor's; apply: of X after the round that begins with the step
    } step[32];
    float x;
};

struct OrthoArgs {
    const OrthoMatrix *list;            // of the group
    int count;
    char *workspace;
    double *squares;                    // [pieces of the group]
    float a, b, c;
    float up_x;                         // what X is held times as it is laid out
    float up_gram, up_factor;           // likewise A and its factor of the step
    float less;                         // from the operands' scales to the result's (kOrthoApply, last: to none)
    const OrthoTile *tiles;             // of the product
    int64_t count_tiles;
    int xt;                             // which of the two transposes is X's
    int step, last;                     // step: 0 or 1 of a round (kOrthoApply: its last); last: the result goes to dst
};

// Matrices that one workgroup takes as a whole: X's blocks and three matrices of p x p in LDS.
constexpr int kOrthoSmallP = 64, kOrthoSmallW = 384;
constexpr int kOrthoSmallLds = 3 * 16384 + kOrthoSmallW / 32 * 8192;
hipError_t gbt_launch_ortho_small(hipStream_t stream, const OrthoArgs &a, const OrthoSmallScales &up, int steps, int together);

enum OrthoProduct { kOrthoGram, kOrthoFactor, kOrthoBetween, kOrthoTotal, kOrthoNext, kOrthoApply };

hipError_t gbt_launch_ortho_begin(hipStream_t stream, const OrthoArgs &a, int64_t pieces, int64_t fill_tiles);
// a.tiles are those of symmetric products' upper halves, or all of X's for kOrthoApply.
hipError_t gbt_launch_ortho_product(hipStream_t stream, const OrthoArgs &a, OrthoProduct product, int num_cu);
