// The 4-bit paged key / value cache: its layout, and what its kernels share.
//
// A page holds page_size tokens (16 .. 256, a power of two).  For each kv head it has one block of
// page_size * (head_dim + 8) bytes, head_dim 64 or 128:
//   key codes     page_size rows of head_dim / 2 bytes; element j of a row is the nibble at bits [4j, 4j + 4) of the row's
//                 little-endian bit stream
//   value codes   for every four tokens 16 runs of head_dim / 64 fours of halfwords, one halfword a token: halfword (run r, part f,
//                 token t) holds elements r * head_dim / 16 + 4 f + 0 .. 3 of token t.  A lane of a matrix-core operand wants
//                 the same elements of four tokens at once: here they are one load, two tokens to a dword, and a token's
//                 own bytes are still its own, so that tokens can be appended without reading what is there.
//   key parameters, value parameters   page_size dwords each: step in the low half, centre in the high half, bfloat16
// An element is (code - 7.5) * step + centre, code 0 .. 15.  bfloat16 parameters: 136 and not 144 bytes a token of 128 (what a
// decode step is bound by), and no overflow where fp16 has one; codes are taken against the rounded parameters, so that the
// rounding of the step (2^-9) costs at most 0.03 of a step at the ends of the range, and that of the centre - near zero for
// rotated rows, where the row's minimum would not be - less.
#pragma once
#include "rotq_internal.h"

namespace rq {

struct Kv4 {
    uint8_t* data;
    int64_t pages;
    int64_t page_bytes;
    int kv_heads, head_dim, page_shift;
};

struct Kv4Append {
    const void *k, *v;
    int dtype;
    int64_t tokens;
    int64_t k_token, k_head, v_token, v_head;     // strides in elements
    const int64_t* slots;
    float clip;
    bool rotate;
};
int kv4_append(const Kv4& c, const Kv4Append& a, hipStream_t s);

struct Kv4Read {
    void *k, *v;                                  // rows x kv_heads x head_dim, contiguous
    int dtype;
    int64_t rows;
    const int64_t* slots;
    bool rotate;
};
int kv4_read(const Kv4& c, const Kv4Read& a, hipStream_t s);

int kv4_copy_pages(const Kv4& c, int layers, int64_t layer_bytes, const int32_t* src, const int32_t* dst, int64_t pairs, hipStream_t s);

struct Kv4Attention {
    const void* q;
    void* o;
    float* lse;
    int dtype;
    int tokens, heads, batch, width;
    int64_t q_token, q_head, o_token, o_head;     // strides in elements
    const int32_t *table, *kv_lens, *q_start;
    float scale;
    bool causal, rotate;
    int window;                                   // 0: none
    int64_t max_len;                              // no sequence is longer
};
size_t kv4_attention_workspace(const Kv4& c, const Kv4Attention& a, int num_cu);
rq_kv4_plan_t kv4_attention_plan(const Kv4& c, const Kv4Attention& a, int num_cu);
int kv4_attention(const Kv4& c, const Kv4Attention& a, int num_cu, float* workspace, hipStream_t s);


// What sequences share: `groups` groups of sequences that stand side by side.
struct Kv4Prefix {
    const int32_t *table, *lens, *group_start;    // [groups][width], [groups], [groups + 1] (sequences)
    int groups, width;
    int64_t max_len;
};
size_t kv4_prefix_workspace(const Kv4& c, const Kv4Attention& a, const Kv4Prefix& p, int num_cu);
rq_kv4_prefix_plan_t kv4_prefix_plan(const Kv4& c, const Kv4Attention& a, const Kv4Prefix& p, int num_cu);
int kv4_prefix_attention(const Kv4& c, const Kv4Attention& a, const Kv4Prefix& p, int num_cu, float* workspace, hipStream_t s);

// Attention that positions have received, added up (q, lse, table ... of `a`; its o is not looked at).
struct Kv4Weights {
    Kv4Attention a;
    float* weights;                               // [batch][kv_heads][positions]
    int64_t w_seq, w_head;                        // strides
    float decay;
};
size_t kv4_weights_workspace(const Kv4& c, const Kv4Attention& a, int num_cu);
int kv4_weights(const Kv4& c, const Kv4Weights& w, int num_cu, void* workspace, hipStream_t s);

struct Kv4Select {
    const float* weights;                         // [layers][batch][kv_heads][n]
    int64_t w_layer, w_seq, w_head;
    const int32_t* kv_lens;
    int layers, batch, kv_heads, n, keep, sinks, recent;
    int32_t* index;                               // [layers][batch][kv_heads][keep]
};
int kv4_select(const Kv4Select& a, hipStream_t s);

struct Kv4Evict {
    const int32_t *index, *table, *new_table;     // new_table null: in place
    float* weights;                               // or null
    int64_t w_layer, w_seq, w_head, layer_bytes;
    int layers, batch, keep, width, new_width, n;
};
int kv4_evict(const Kv4& c, const Kv4Evict& a, hipStream_t s);

}  // namespace rq
