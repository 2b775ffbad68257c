// How the gradient of an embedding is cut up (functions of the sizes alone).
#pragma once

#include "common.cuh"

namespace sbp {

struct EmbeddingPlan {
    int passes;             // of the sort, 8 bits each
    int tile, tiles;        // tokens of a block of the sort, blocks
    int chunk, chunks;      // entries of the sorted list that are summed by one block, blocks
};
EmbeddingPlan embedding_plan(int64_t n, int64_t vocab, int64_t d);

}  // namespace sbp
