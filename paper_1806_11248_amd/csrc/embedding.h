// What the embedding kernels and their entry points share.
#pragma once

#include "gbt_internal.h"

struct EmbedArgs {
    const void *ids;
    int id_bytes;                      // 4 or 8
    int width, log_lanes, slabs;       // a row's columns are taken in slabs of 8 << log_lanes, by 1 << log_lanes lanes
    int vector;                        // rows can be read and written 8 elements at a time
    int64_t n_ids, n_rows;
    int64_t table_stride, out_stride;  // elements
    float scale;
    const void *table;                 // [n_rows]; the gradient where that is computed
    void *out;                         // [n_ids]; its gradient likewise
    int table_dtype, out_dtype;
    // backward
    int accumulate;
    int chunk, chunks;                 // sorted places that a group of lanes adds up
    const uint32_t *key, *pos;         // sorted ids (n_rows: outside the table) and their places
    float *part;                       // [chunks][2][slabs * (8 << log_lanes)]: sums of runs that go on in other chunks
    int zero_rows;                     // rows that a workgroup of the few-ids kernel owns, or that a wave clears
    // backward, few rows: a wave adds up `chunk` places, part is [chunks][n_rows][8 << log_lanes]; one slab
    uint32_t *seen;                    // [chunks]: the rows that it met, a bit for each
};

constexpr int kEmbedFewIds = 2048;     // more than that are sorted, or added up in LDS
constexpr int kEmbedFewRows = 32;      // up to so many are added up in LDS, unsorted
constexpr int kSortItems = 4096;       // ids that a workgroup of the sort ranks at a time
constexpr int kSortTiles = 256;        // workgroups of a pass at most
constexpr int kSortDigits = 1024;      // of a pass at most

struct SortPass {
    const void *ids;                   // of the first pass, else NULL
    int id_bytes;
    const uint32_t *key_in, *pos_in;
    uint32_t *key_out, *pos_out, *hist;
    int64_t n, n_rows, tile;           // tile: ids of a workgroup, a multiple of kSortItems
    int tiles, shift, bits;
};

hipError_t gbt_launch_embedding(hipStream_t stream, const EmbedArgs &a);
hipError_t gbt_launch_sort_pass(hipStream_t stream, const SortPass &p);
hipError_t gbt_launch_embedding_grad(hipStream_t stream, const EmbedArgs &a);       // of sorted ids
hipError_t gbt_launch_embedding_grad_rows(hipStream_t stream, const EmbedArgs &a);  // of few rows
hipError_t gbt_launch_embedding_grad_few(hipStream_t stream, const EmbedArgs &a);
