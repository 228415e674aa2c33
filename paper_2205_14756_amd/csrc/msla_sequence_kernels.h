// Host-side launch interfaces of the sequence operators' kernels (validated arguments, everything decided).
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace msla {

struct RecurrenceRows {
    void* p;
    long ts, hs;
};

// How a call is cut into segments, and where its workspace keeps what (byte offsets).
struct RecurrencePlan {
    int segment = 0, slots = 0;
    bool cut = false;               // more than one segment to a sequence is possible
    size_t d_states_at = 0, decay_at = 0, d_decay_at = 0, crossing_at = 0, dots_at = 0, last_at = 0, bytes = 0;
};

struct RecurrenceCall {
    int what;                       // 0 forward, 1 backward, 2 one token a sequence
    RecurrencePlan plan;
    int sequences;
    long tokens;
    const int* offsets;
    int heads_q, heads_kv, head_dim, rectify;
    float scale;
    RecurrenceRows q, k, v, out, d_out, d_q, d_k, d_v;
    const void* gate;
    long gate_ts;
    const float* initial;
    float* final_state;
    const float* d_final;
    void* d_gate;
    long d_gate_ts;
    float* d_initial;
    char* ws;
};

hipError_t launch_recurrence(int dt, const RecurrenceCall& call, hipStream_t stream);

struct NormCall {
    const void *x, *residual, *weight;
    void *y, *sum;                  // y: the storage type, or e4m3 where `scale` is given
    float* scale;
    int64_t rows;
    int channels;
    float eps;
    bool plain;                     // y = r: no norm, no weight (rows into 8 bits)
};
hipError_t launch_norm(int dt, const NormCall& call, hipStream_t stream);

int norm_backward_blocks(int64_t rows, int channels, int elem);
hipError_t launch_norm_backward(int dt, const void* sum, const void* weight, const void* d_y, const void* d_sum, void* d_r, float* d_weight,
                                float* partials, int64_t rows, int channels, float eps, hipStream_t stream);

hipError_t launch_linear_quantized(int dt, const void* x8, const float* x_scale, const void* w8, const float* w_scale, void* y, int64_t rows,
                                   int c_in, int c_out, hipStream_t stream);

}  // namespace msla
