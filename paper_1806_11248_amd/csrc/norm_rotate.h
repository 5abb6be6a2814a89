// What the kernels of head norms with rotation and their entry points share.
#pragma once

#include "gbt_internal.h"
#include "heads.h"

struct RotateArgs {
    AttnView q, k, v, q_out, k_out, v_out;   // v: data is NULL where there is none
    AttnView dq, dk;                         // backward: the gradients of q_out and k_out are in q_out and k_out
    const int64_t *q_ptr, *k_ptr;            // NULL: sequences of one length
    const int32_t *k_len;                    // NULL: all of a slot
    const void *positions;                   // NULL: the place in the sequence
    int position_bytes;
    const float *q_weight, *k_weight;        // NULL: ones
    const double *turns;
    int64_t rows, out_rows;                  // of q, k and v; of k_out and v_out
    int n_seq, heads, kv_heads;
    int dim, turned, halves, store, slots;   // slots: positions are counted from the end of what k_ptr or k_len say is in use
    float eps;
    int log_lanes;                           // 1 << log_lanes lanes for a line, of which dim / 8 work
    int row_group;                           // rows that a wave takes side by side
    int parts;                               // forward: a row's heads are shared by so many waves
    int blocks;
    int k_row_group, q_blocks;               // backward: rows of k side by side; workgroups for q, the others take k
    float *part;                             // [blocks][128]: the weights' gradients
    float *dq_weight, *dk_weight;
};
constexpr int kRotateDim = GBT_MAX_HEAD_DIM;

hipError_t gbt_launch_norm_rotate(hipStream_t stream, const RotateArgs &a, int dtype);
hipError_t gbt_launch_norm_rotate_grad(hipStream_t stream, const RotateArgs &a, int dtype);
