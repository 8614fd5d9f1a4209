// Products of compressed matrices with a few vectors: what the decoder's file offers to the layer's.  A wave multiplies the values of its
// stream as it decodes them and leaves one sum per matrix row that the stream touches (a piece of the row) and vector; nothing of the matrix goes to memory.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "zipmoe.h"
#include "zipmoe_product_rule.h"

namespace zipmoe {

// Which vectors meet which matrix, and where the sums go.
struct ProductCall {
    const int32_t *ids;        // DEVICE [n_pairs]: the expert of every pair of a token and an expert
    const uint16_t *x;         // DEVICE bf16 rows
    const uint16_t *rest;      // what is to be added to them, rows alike; or null
    float *sums;               // DEVICE [matrices of an expert, n_pairs, pieces]
    int64_t x_stride;
    uint32_t n_pairs, top_k;
    uint32_t by_pair;          // a row of x for every pair, else for every token
    uint32_t width;            // values of a matrix row, a multiple of eight
    uint32_t pieces;
};

// Multiplies n matrices; matrix i is number i % per_expert of expert ids[i / per_expert].  Checked by the caller: addresses, and product_fits.
int product_launch(const void *const *blobs, const uint64_t *const *tables, const zm_tensor_info *const *infos, const int32_t *ids, int n, int per_expert,
                   const ProductCall &call, hipStream_t stream);

}  // namespace zipmoe
