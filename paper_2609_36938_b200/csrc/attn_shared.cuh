// Arguments of janus_attn_decode_shared, checked, as its two routes take them.
#pragma once

#include "janus_common.cuh"

namespace janus {

struct SharedAttnArgs {
    const void* q;
    int B, H_q, d_qk;
    const void* k_pool;
    int64_t k_page_stride, k_tok_stride, k_head_stride;
    const void* v_pool;
    int64_t v_page_stride, v_tok_stride, v_head_stride;
    int n_kv_heads, d_v, page_size;
    int64_t n_phys_pages;
    const int32_t* prefix_table;
    int64_t prefix_len;
    const int32_t* page_tables;
    const int64_t* table_offsets;
    const int64_t* kv_lens;
    int64_t max_len;
    float softmax_scale;
    void* out;
    float* lse;
    void* ws;
    int32_t* dev_status;
};

bool attn_shared_tc_supported(int d_qk, int d_v);
size_t attn_shared_tc_workspace(int B, int H_q, int n_kv_heads, int d_v, int64_t prefix_len, int64_t max_len);
int launch_attn_shared_tc(const SharedAttnArgs& a, cudaStream_t stream);

}  // namespace janus
