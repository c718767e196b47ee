// What the kernels of pbs_decode_attn share.
#pragma once
#include "pbs_host.h"
#include "serving.h"

namespace pbs {

constexpr int kPrefixRows = 128;                           // rows of a workgroup of the kernel for many rows

struct DecodeArgs {
    int n_seq, q_len, h_q, h_kv, r;
    int page_log, pages, max_pages, max_len, prefix_len;
    int row_tiles;                                         // of a sequence's q_len * r rows
    int units;                                             // of a sequence: h_kv * row_tiles
    int shares;                                            // waves of the own keys
    int slot_rows;                                         // rows of a piece in the workspace
    int p_chunk, p_parts, p_row_tiles;                     // the same of the prefix
    float c2;                                              // scale * log2(e)
    pbs_strides q, o;
    const bf16_t *Q;
    const uint8_t *K, *V;
    const float *kf, *vf;
    const int32_t *table, *lens, *prefix;
    bf16_t *O;
    float *lse, *part_o, *part_ml, *piece_o, *piece_ml;
    int2 *pieces;                                          // of a unit: its first slot and how many
    // many rows over an 8-bit cache: the prefix's values as bf16 [h_kv][p_room][d], its factors [h_kv][p_room]
    int p_room;
    bf16_t *line_k, *line_v;
    float *line_kf, *line_vf;
};

// The prefix against more rows than a wave of decode_attn.hip takes (prefix_attn.hip).  Always into the workspace: it may read
// its queries twice, and O may be Q.
pbs_status launch_prefix(const DecodeArgs &a, int dtype, int d, hipStream_t s);

}  // namespace pbs
