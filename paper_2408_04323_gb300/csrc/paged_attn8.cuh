// What the two kernels of attention over an 8-bit cache share.
#pragma once

#include <cuda.h>

#include "internal.h"

struct Attn8Args {
    int32_t bs_log, n_heads, n_kv_heads, group, n_req, causal, window, max_new;
    int32_t few;               // requests of up to so many tokens are the rows kernel's, the others the tiles kernel's
    int32_t toks;              // rows kernel: tokens of an item
    int32_t share;             // rows kernel: heads that as many warps take together
    int64_t n_tokens, n_blocks;
    const int32_t* query_start;
    const int32_t* kv_len;
    const int32_t* table;
    int64_t ld_table;
    const uint16_t* q;
    int64_t q_ld_token, q_ld_head;
    const uint8_t* k;
    const uint8_t* v;
    int64_t ld_block, ld_token, ld_head;
    const float* k_scale;
    const float* v_scale;
    float scale_log2;
    uint16_t* out;
    int64_t out_ld_token, out_ld_head;
    float* lse;
    float* parts;              // two per warp, then two per block
    uint32_t* warp_count;      // arrivals per split item, by its first warp, zero between calls
    uint32_t* block_count;     // likewise of blocks
    float* tile_parts;         // the tiles kernel's
    uint32_t* tile_count;
    uint32_t* err;
};

// The tiles kernel (paged_attn.cu): requests of more than args.few tokens.  Its workspace, per multiprocessor.
scoot_status scoot_attn8_tiles(scoot_ctx* ctx, const scoot_kv_layout* layout, const Attn8Args& args, bool bf16, int sms, cudaStream_t st, bool beside);
size_t scoot_attn8_tile_bytes(int head_dim);
// The map of an 8-bit cache: boxes of up to `tokens` tokens of a block and head, rows of head_dim bytes swizzled by their size.
bool scoot_encode_codes(CUtensorMap* map, const scoot_kv_layout* layout, const void* cache, int tokens);
