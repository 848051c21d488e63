// What stands between a decoder layer's blocks: residual sums with the norms around a block, rotary positions (pop_block.hip).
// Launchers: arguments have been checked; each returns the launch's status.
#pragma once
#include "pop_internal.h"

namespace pop {

struct BlockNormArgs {
    const void *x;  // residual stream
    int x_bf16;
    long long x_stride;
    const void *u;  // a block's output, NULL for none
    int bf16;       // of u, gate, weights and z
    long long u_stride;
    const void *gate;  // NULL for none
    long long gate_stride;  // 0 for one row
    const void *w_post, *w_pre;
    int n, d, post;
    float offset, eps, x_scale, u_scale;
    void *x_out;
    long long x_out_stride;
    void *z;
    long long z_stride;
};
hipError_t launch_block_norm(const BlockNormArgs &a, hipStream_t s);

struct RotaryArgs {
    const void *q, *k;
    int bf16, n, n_heads, n_kv, d, r, pairs;
    long long q_stride, k_stride;
    const int *positions;
    const double *turns;
    float amplitude;
    void *q_out, *k_out;
    long long q_out_stride, k_out_stride;
};
hipError_t launch_rotary(const RotaryArgs &a, hipStream_t s);

constexpr int kMostNormWidth = 65536;  // channels that the largest workgroup holds in registers
constexpr int kMostRotary = 1024;      // channels of a head that are turned: a token's angles stand in LDS

}  // namespace pop
