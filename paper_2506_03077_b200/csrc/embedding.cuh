// How the gradient of an embedding is cut up (functions of the sizes alone).
#pragma once

#include "common.cuh"

namespace sbp {

struct EmbeddingPlan {
    int passes;             // of the sort
    bool one_launch;        // of the sort, in a cluster
    int tile, tiles;        // else: tokens of a block of the sort, blocks
    int chunk, chunks;      // entries of the sorted list that are summed by one block, blocks
    int partial_width;      // floats of a row of partial sums
};
EmbeddingPlan embedding_plan(int64_t n, int64_t vocab, int64_t d);
int embedding_counts(const EmbeddingPlan &p);      // ints the sort's launches hand on
int embedding_cap_sort(int blocks);                // of a cluster of the sort at most (a test's); returns what it was

}  // namespace sbp
