// Host-side launch interfaces of the kernels of a selective state space layer (validated arguments, everything decided).
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "slots.h"

namespace msla {

struct TokenRows {
    void* p;
    int64_t ts;                     // elements from row to row
};

struct ScanCall {
    int channels, groups, states, softplus;
    Slots slots;
    bool cut;                       // more than one slot to a sequence is possible
    TokenRows x, delta, b, c, gate, out, d_out, d_x, d_delta, d_b, d_c, d_gate;
    const float *a, *skip, *bias, *initial, *d_final;
    float *final_state, *d_a, *d_skip, *d_bias, *d_initial;
    // workspace: a slot's own state and, behind the join, the one that it starts from; the sum of its steps; the same for the state's gradient
    float *states_at, *steps_at, *d_states_at;
    // the gradient's marks: the states in front of every scan_lanes() tokens of a sequence (of a slot from zero, with the steps so far, where it is cut)
    Slots marks;
    float *marks_at, *mark_steps_at;
    // parts of the sums over tokens (a slot's, [channels, states + 2]) and over channels (a tile's, [tokens, 2 * states])
    float *parts_at, *shared_at;
};

constexpr int kScanSlice = 32;      // channels of a workgroup, of one group
inline int scan_tiles(int channels, int groups) { return groups * ((channels / groups + kScanSlice - 1) / kScanSlice); }
inline int scan_lanes(int states) { return states == 8 ? 8 : 16; }     // that share a channel; tokens from mark to mark of the gradient, a quarter of a tile's

hipError_t launch_scan_forward(int dt, const ScanCall& c, hipStream_t stream);
hipError_t launch_scan_backward(int dt, const ScanCall& c, hipStream_t stream);
hipError_t launch_scan_step(int dt, const ScanCall& c, hipStream_t stream);

struct ConvCall {
    int channels, width, silu;
    Slots slots;
    TokenRows x, out, d_out, d_x;
    const void *weight, *bias, *initial, *d_final;
    void *final_state, *d_initial;
    float *d_weight, *d_bias, *parts_at;
};
hipError_t launch_conv_forward(int dt, const ConvCall& c, hipStream_t stream);
hipError_t launch_conv_backward(int dt, const ConvCall& c, hipStream_t stream);
hipError_t launch_conv_step(int dt, const ConvCall& c, hipStream_t stream);

struct LayerNormCall {
    const void *x, *residual, *weight, *bias;
    void *y, *sum;
    int64_t rows;
    int channels;
    float eps;
};
hipError_t launch_layer_norm(int dt, const LayerNormCall& c, hipStream_t stream);
int layer_norm_blocks(int64_t rows, int channels, int elem);       // workgroups of the gradient, and parts of d_weight and d_bias
hipError_t launch_layer_norm_backward(int dt, const void* sum, const void* weight, const void* d_y, const void* d_sum, void* d_r, float* d_weight,
                                      float* d_bias, float* parts, int64_t rows, int channels, float eps, hipStream_t stream);

hipError_t launch_quantize_integer(int dt, const void* x, void* x8, float* scale, int64_t rows, int channels, hipStream_t stream);
hipError_t launch_linear_integer(int dt, const void* x8, const float* x_scale, const void* w8, const float* w_scale, void* y, int64_t rows, int c_in,
                                 int c_out, hipStream_t stream);

// The sums over `count` parts, `stride` floats apart, in a fixed order: of the first n[0] columns to out[0], of the n[1] behind them to out[1],
// of the n[2] behind those to out[2] (NULL: not wanted).
struct PartSums {
    float* out[3];
    int64_t n[3];
};
hipError_t launch_sum_parts(const float* parts, int64_t count, int64_t stride, const PartSums& to, hipStream_t stream);

}  // namespace msla
