// Attention of one new token over a paged key-value cache, and the copy of a prompt into its pages.
#pragma once
#include "common.cuh"

namespace based {

struct PagedCall {
    const void *q, *k, *v;                 // [B,Hq,d], [B,Hk,d]
    void *k_pages, *v_pages;               // row (page, head, slot) at page * page_stride + head * head_stride + slot * token_stride, elements
    long long page_stride, head_stride, token_stride;
    const int *table, *pos;                // [B,max_pages], [B]
    const float* slopes;                   // [Hq] or null
    void* out;                             // [B,Hq,d]
    int B, Hq, Hk, d, pages, page_size, max_pages, window;     // window 0: all
    float scale, cap;                      // cap 0: none
};
size_t paged_decode_bytes(int B, int Hq, int Hk, int d, int page_size, int max_pages, based_dtype io);
based_status launch_paged_decode(const PagedCall& c, void* workspace, based_dtype io, cudaStream_t stream);

struct PagedWrite {
    based_heads k, v;                      // [B,H,L,d]
    void *k_pages, *v_pages;
    long long page_stride, head_stride, token_stride;
    const int *table, *pos, *counts;       // counts [B] or null: L
    int B, H, L, d, pages, page_size, max_pages;
};
based_status launch_paged_write(const PagedWrite& c, based_dtype io, cudaStream_t stream);

}  // namespace based
