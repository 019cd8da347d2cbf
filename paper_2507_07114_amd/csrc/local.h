// Internal interface between the C ABI of the local-gradient operators
// (local_api.cpp) and their HIP kernels (local_embed.hip, local_act.hip,
// local_wgrad.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lossy {

constexpr int kActGroup = 32;   // columns of a token that share a scale
constexpr int kActMinExp = -117;  // smallest exponent of a scale

// A token batch: [n][ld] ids of 4 or 8 bytes, and where each worker's ends.
struct TokenView {
    const void* ids;
    int64_t ld;
    int64_t first, v;  // held ids are [first, first + v)
    int wide;          // 64-bit ids
};

// Activation rows [n][t][ld].
struct ActView {
    void* p;
    int64_t ld;
    int bf16;
};

// A table or weight [rows][h] at element `offset` of every row of [n][ld].
struct RowView {
    void* p;
    int64_t ld, offset;
    int bf16;
};

// 8-bit checkpoint: codes [n][t][ld_q], exponent bytes [n][t][ld_s].
struct PackView {
    uint8_t* q;
    int64_t ld_q;
    uint8_t* s;
    int64_t ld_s;
};

struct EmbedParams {
    int n;
    int64_t t, h;
    const int32_t* lengths;
    TokenView tok;
    RowView table;
    float scale;
    ActView out;
};

struct EmbedGradParams {
    int n;
    int64_t t, h;
    const int32_t* lengths;
    TokenView tok;
    ActView dy;
    float scale;
    RowView grads;
    int accumulate;
};

struct PackParams {
    int n;
    int64_t t, h;
    const int32_t* lengths;
    ActView x;  // ll_act_pack: input; ll_act_unpack: output
    PackView c;
};

struct WgradParams {
    int n;
    int64_t t, o, h;
    const int32_t* lengths;
    ActView dy;
    PackView x;
    float scale;
    RowView grads;
    int accumulate;
};

hipError_t launch_embed(const EmbedParams& p, hipStream_t s);
hipError_t launch_embed_grad(const EmbedGradParams& p, void* ws, hipStream_t s);
size_t embed_grad_workspace(int64_t n, int64_t t, int64_t h, int64_t v);
hipError_t launch_act_pack(const PackParams& p, hipStream_t s);
hipError_t launch_act_unpack(const PackParams& p, hipStream_t s);
hipError_t launch_act_wgrad(const WgradParams& p, void* ws, hipStream_t s);
size_t act_wgrad_workspace(int64_t n, int64_t t, int64_t o, int64_t h);

}  // namespace lossy
