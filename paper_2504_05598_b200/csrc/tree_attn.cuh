// What the two forms of del_tree_attention share: arguments, a sequence's view of its row, the host's launch interface.
#pragma once

#include "pages.cuh"

struct TreeArgs {
    PageView kv;
    const bf16 *q;
    bf16 *out, *out_lo;
    const int32_t *table, *lens, *nodes;
    const uint64_t *mask;
    int32_t *err;              // may be null
    int64_t q_seq, q_node, o_seq, o_node;
    int32_t max_nodes, nh, layer, cols, stride;
    float scale;               // times log2(e)
};

namespace tree {

// what a CTA knows of its sequence
struct Seq {
    int len, n, n_keys;        // committed positions, nodes, positions that may be seen (cut at the table's end)
    const int32_t *pt;
};

__device__ __forceinline__ Seq load_seq(const TreeArgs &a, int b) {
    Seq s;
    const int cap = a.cols * 16;
    s.len = min(max(a.lens[b], 0), cap);
    s.n = a.nodes ? min(max(a.nodes[b], 0), a.max_nodes) : a.max_nodes;
    s.n_keys = min(s.len + s.n, cap);
    s.pt = a.table + (size_t)b * a.stride;
    return s;
}

// bits of the nodes that node i of sequence b sees
__device__ __forceinline__ uint64_t node_bits(const TreeArgs &a, int b, int i) {
    return a.mask ? a.mask[(size_t)b * a.max_nodes + i] : (2ull << i) - 1;
}

__device__ __forceinline__ bool sees(uint64_t bits, int tok, int len, int n_keys) {
    const int j = tok - len;
    return tok < n_keys && (j < 0 || ((bits >> j) & 1));       // (n_keys - len <= 64)
}

// two outputs: packed high and low parts; where the high part is infinite the low one is zero (the difference would be no number)
__device__ __forceinline__ void split_out(float x0, float x1, uint32_t &hi, uint32_t &lo) {
    split_bf16x2(x0, x1, hi, lo);
    if ((hi & 0x7fffu) == 0x7f80u) lo &= 0xffff0000u;
    if ((hi & 0x7fff0000u) == 0x7f800000u) lo &= 0x0000ffffu;
}

}  // namespace tree

// del_tree_attention behind its checks.  max_len: what lens are expected to reach; streaming: register-streaming GEMMs run around it (tree_form.h).
cudaError_t launch_tree_attention(const TreeArgs &a, int batch, int max_len, cudaStream_t st, bool streaming);
// Tiles of up to 256 query rows on tcgen05 (tree_attn_tc.cu)
cudaError_t launch_tree_attention_tc(const TreeArgs &a, int batch, int max_len, cudaStream_t st);
