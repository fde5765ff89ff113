// What the kernels of ragged attention (attn_ragged.hip) and their host side (aed_train.hip) share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace aed {

struct AttnTensor {  // element (row, head, column) at p + row * row_pitch + head * head_pitch + column * element size
    char* p;
    int64_t row, head;  // bytes
};

// A workgroup's share for every head.  Forward and query gradients: `rows` query rows from q_row on against keys k_begin .. k_end - 1 of
// the sequence whose keys begin with row k_row; pos: which key the first row stands at (k_len - q_len + its number, may be negative).
// Key gradients: `rows` keys from k_row on against query rows k_begin .. k_end - 1 of the sequence whose queries begin with q_row;
// pos: the first key's place less k_len - q_len, that is the query row that stands at it.
// part >= 0: the keys are only a part of the row's, sums and maxima go to that place.
struct RaggedItem {
    int64_t k_row;
    int32_t q_row, rows, pos, k_begin, k_end, part;
};
struct RaggedJoin {  // rows whose parts are to be added up
    int32_t q_row, rows, part, n_parts;
};

struct RaggedArgs {
    AttnTensor q, k, v, o, d_o, dq, dk, dv;
    float* lse;              // [rows, heads]
    const uint8_t* key_mask;  // by key row; nullptr: all keys are seen
    const char* zeros;       // 512 bytes
    const void* bias;        // [buckets, heads], in the tensors' type
    const uint8_t* bucket_of;  // [span], by key - query + max_distance
    const int2* bucket_range;  // [buckets]: first of a bucket's places with the margins on both sides, and one past its last
    float* delta;            // [rows, heads]: sum over a row of gradient times output
    float* part_o;           // [part, heads, tile rows, D]
    float2* part_ml;         // [part, heads, tile rows]: maximum (of scores times log2 e) and sum
    float2* large;           // [rows, heads], with a bias, of rows with a large lse: maximum of the scores times log2 e, log2 of the weights' sum
    float* part_bias;        // [item, heads, buckets]
    const RaggedItem* items;
    int n_items;
    int bias_items;          // items that part_bias has sums of
    void* d_bias;            // [buckets, heads]
    const RaggedJoin* joins;
    float scale;
    int heads, share;        // share: query heads to a key head
    int causal, buckets, max_distance, span;
};

constexpr int kAttnRows = 128;  // query rows of an item of many, keys of an item of key gradients
constexpr int kAttnPair = 64;   // the same where wavefronts share rows or keys in pairs
constexpr int kAttnFew = 32;    // and of few (attn_few_kernel)
constexpr int kAttnMargin = 72;  // places of the bias in LDS beyond both ends of its range
constexpr int kAttnMaxPitch = 0x40000000 / 64 - 64;  // bytes between rows: 64 of them stay below 2^30, and twice that in 32 bits

// Each returns hipSuccess or what the launch reported.  tile_rows: query rows of an item.
hipError_t launch_attn_forward(const RaggedArgs& a, int head_dim, bool bf16, int tile_rows, hipStream_t s);
hipError_t launch_attn_join(const RaggedArgs& a, int head_dim, bool bf16, int tile_rows, int joins, hipStream_t s);
hipError_t launch_attn_dq(const RaggedArgs& a, int head_dim, bool bf16, int tile_rows, hipStream_t s);
// and the bias's gradient from what dq's launch left
hipError_t launch_attn_dkv(const RaggedArgs& a, int head_dim, bool bf16, int tile_keys, hipStream_t s);

}  // namespace aed
