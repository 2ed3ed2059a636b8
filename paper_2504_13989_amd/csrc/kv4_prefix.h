// How a call of rq_kv4_prefix_attention is laid out (kernels_kv4_prefix.hip), and its launches of the kernel for many rows.
#pragma once
#include "kv4_attention.h"

namespace rq {

struct PrefixPlan {
    bool separate;                                // each sequence takes prefix and own positions in one launch
    int waves;                                    // of a workgroup then
    bool many, own_many;                          // kernel for many rows: for the prefixes, for what is behind them
    int groups;                                   // of waves that share a workgroup's keys
    int own_copies;                               // kernel for few rows: copies of a sequence's rows among the columns
    int shared_tiles, own_tiles;                  // row tiles at most
    int shared_chunk, shared_chunks, own_chunk, own_chunks;   // keys of a workgroup, chunks of a row tile
    int slice;                                    // tokens that the workspace holds partial results of: those of a call are taken in turns
    size_t bytes;                                 // workspace
};

void launch_prefix_many(const PrefixJob& job, Part part, int groups, hipStream_t s);

}  // namespace rq
