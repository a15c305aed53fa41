// Shared by the layer of experts (expert_layer.hip) and its host code (f8_host.cpp).
#pragma once
#include "f8.h"

namespace bitstack {

constexpr int kLayerTokens = 64;   // at most: the tokens of an expert are a 64-bit mask

struct LayerExpert {   // that has tokens
    int expert, base;   // base: their first row; rows are sorted by expert, then token
    unsigned long long tokens;
};
// Choices by sizes alone
struct LayerPlan {
    int fragments;   // of 16 tokens in a unit of work; an expert with more tokens has several
    int most;        // entries of the list of experts, at most
    int up_few;      // k_layer_up: eight gates to a unit, not 16
    int pack;        // k_layer_down: the parts of h are columns of one fragment
    int down_rows, tiles_down, splits;   // k_layer_down: rows of W2 in a tile, tiles, parts of the columns
};
LayerPlan layer_plan(int tokens, int hidden, int width, int experts, int top_k, bool f32);   // f32: x

struct LayerParams {
    const void* x;
    const void* logits;
    const unsigned char* w1;   // [experts][2 width] rows of e4m3
    const unsigned char* s1;
    const unsigned char* w2;   // [experts][hidden]
    const unsigned char* s2;
    const void* residual;      // or null
    void* y;
    size_t ld_x, ld_logits, ld_w1, ld_w2, ld_r, ld_y;   // elements, of the weights bytes
    int dtype, logits_dtype, s1_f32, s2_f32;
    int tokens, top_k, renormalise, experts, hidden, width;
    int fragments, most, up_few, pack;   // LayerPlan
    // workspace
    int* count;                // entries of list
    LayerExpert* list;         // [most]
    float* row_weight;         // [rows]
    unsigned char* row_token;  // [rows]
    unsigned* arrived;         // [tiles_down]
    unsigned short* h;         // bf16 parts of h, in the order in which k_layer_down loads them
    float* part;               // [tiles_down][splits][tokens][down_rows]
    unsigned h_bytes;
    int h_parts;
    int down_rows, tiles_down, splits;
};
hipError_t launch_expert_layer(const LayerParams& p, hipStream_t st);

}  // namespace bitstack
