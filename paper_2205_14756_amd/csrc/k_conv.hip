// The short causal convolution of each channel with its own taps, over sequences: pre_i = bias + sum_k w[k] x_{i - width + 1 + k}, out = pre or silu(pre).
//
// Bound by memory.  A thread has a piece of 16 bytes of the channels and a run of tokens of one sequence (a slot), whose last width - 1 rows stay in registers as the
// run goes on; those before the run are read once more (out of a cache).  The sequence's state is those rows: the ones in front of its first
// token, and the last ones.
//
// The gradient goes over the same runs and the width - 1 tokens behind them, whose part of d_x it needs: pre again, d_pre = d_out silu'(pre), d_x_i = sum_m
// w[width - 1 - m] d_pre_{i + m}; taps and bias are summed over a run in registers, over runs through parts that a second launch adds up.
#include "msla_device.h"
#include "msla_layer_kernels.h"
#include "norm_rows.h"

namespace msla {
namespace {

constexpr float kLog2e = 1.44269504088896340736f;
__device__ __forceinline__ float sigmoid_of(float v) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2e * v)); }

template <class T>
__device__ __forceinline__ const T* row(const TokenRows& r, int t) { return (const T*)r.p + (int64_t)t * r.ts; }
template <class T>
__device__ __forceinline__ T* row_out(const TokenRows& r, int t) { return (T*)r.p + (int64_t)t * r.ts; }

// A thread's place: `across` lanes (a power of two, 256 at most) take neighbouring pieces of a row, so that a wave reads whole lines.
template <int VEC>
struct Place {
    Piece<VEC> piece;
    int slot;
    __device__ __forceinline__ Place(int channels, int across, int blocks_across)
        : piece((int)(blockIdx.x % blocks_across) * across + (int)(threadIdx.x % across), channels),
          slot((int)(blockIdx.x / blocks_across) * (256 / across) + (int)(threadIdx.x / across)) {}
};

template <class T, int W>
struct Taps {
    float w[W][Traits<T>::kVec], bias[Traits<T>::kVec];
    __device__ __forceinline__ Taps(const ConvCall& c, int at) {
#pragma unroll
        for (int e = 0; e < Traits<T>::kVec; ++e) {
            const bool in = at + e < c.channels;
#pragma unroll
            for (int k = 0; k < W; ++k) w[k][e] = in ? Traits<T>::to_f32(((const T*)c.weight)[(int64_t)(at + e) * W + k]) : 0.0f;
            bias[e] = in && c.bias ? Traits<T>::to_f32(((const T*)c.bias)[at + e]) : 0.0f;
        }
    }
    __device__ __forceinline__ float pre(const float (&rows)[W][Traits<T>::kVec], int e) const {
        float v = bias[e];
#pragma unroll
        for (int k = 0; k < W; ++k) v = fmaf(w[k][e], rows[k][e], v);
        return v;
    }
};

// the width - 1 rows in front of token t of a sequence that starts at lo, oldest first, to rows[0 .. W - 2]
template <class T, int W>
__device__ __forceinline__ void rows_before(const ConvCall& c, const Slot& s, int t, int at, float (&rows)[W][Traits<T>::kVec]) {
    constexpr int kVec = Traits<T>::kVec;
#pragma unroll
    for (int k = 0; k < W - 1; ++k) {
        const int i = t - (W - 1) + k;
        if (i >= s.lo) {
            load_row<T>(row<T>(c.x, i), at, c.channels, rows[k]);
        } else if (c.initial) {
            load_row<T>((const T*)c.initial + ((int64_t)s.sequence * (W - 1) + (W - 1 - (s.lo - i))) * c.channels, at, c.channels, rows[k]);
        } else {
#pragma unroll
            for (int e = 0; e < kVec; ++e) rows[k][e] = 0.0f;
        }
    }
}

template <class T, int W>
__global__ void __launch_bounds__(256) conv_kernel(ConvCall c, int across, int blocks_across, int slots) {
    constexpr int kVec = Traits<T>::kVec, kAhead = 4;
    const Place<kVec> me(c.channels, across, blocks_across);
    if (!me.piece.live || me.slot >= slots) return;
    const Slot s = slot_at(c.slots, me.slot);
    if (!s.used) return;
    const int at = me.piece.at;
    const Taps<T, W> taps(c, at);
    float rows[W][kVec];
    rows_before<T, W>(c, s, s.from, at, rows);
    for (int t0 = s.from; t0 < s.until; t0 += kAhead) {
        typename Traits<T>::Vec raw[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) raw[i] = load_raw<T>(row<T>(c.x, min(t0 + i, s.until - 1)), at, c.channels);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (t0 + i >= s.until) break;
            float out[kVec];
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                rows[W - 1][e] = Traits<T>::to_f32(raw[i][e]);
                const float pre = taps.pre(rows, e);
                out[e] = c.silu ? pre * sigmoid_of(pre) : pre;
#pragma unroll
                for (int k = 0; k < W - 1; ++k) rows[k][e] = rows[k + 1][e];
            }
            store_row<T>(row_out<T>(c.out, t0 + i), at, c.channels, out);
        }
    }
    if (s.last && c.final_state) {
#pragma unroll
        for (int k = 0; k < W - 1; ++k) store_row<T>((T*)c.final_state + ((int64_t)s.sequence * (W - 1) + k) * c.channels, at, c.channels, rows[k]);
    }
}

template <class T, int W>
__global__ void __launch_bounds__(256) conv_backward_kernel(ConvCall c, int across, int blocks_across, int slots) {
    constexpr int kVec = Traits<T>::kVec, kAhead = 4;
    const Place<kVec> me(c.channels, across, blocks_across);
    if (!me.piece.live || me.slot >= slots) return;
    const Slot s = slot_at(c.slots, me.slot);
    const int at = me.piece.at;
    float d_w[W][kVec], d_b[kVec];
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
        d_b[e] = 0.0f;
#pragma unroll
        for (int k = 0; k < W; ++k) d_w[k][e] = 0.0f;
    }
    if (s.used) {
        const Taps<T, W> taps(c, at);
        float rows[W][kVec], d_pre[W][kVec];        // of the last W tokens
        rows_before<T, W>(c, s, s.from, at, rows);
#pragma unroll
        for (int k = 0; k < W; ++k)
#pragma unroll
            for (int e = 0; e < kVec; ++e) d_pre[k][e] = 0.0f;
        const int beyond = s.until + W - 1;
        for (int t0 = s.from; t0 < beyond; t0 += kAhead) {
            typename Traits<T>::Vec raw[kAhead], grad[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int t = min(t0 + i, s.hi - 1);
                if (s.hi > s.lo) {
                    raw[i] = load_raw<T>(row<T>(c.x, t), at, c.channels);
                    grad[i] = load_raw<T>(row<T>(c.d_out, t), at, c.channels);
                } else {
                    raw[i] = grad[i] = typename Traits<T>::Vec{};
                }
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int t = t0 + i, r = t - (W - 1);
                if (t >= beyond) break;
                const bool own = t < s.until, in = t < s.hi;
                float out[kVec];
#pragma unroll
                for (int e = 0; e < kVec; ++e) {
                    rows[W - 1][e] = Traits<T>::to_f32(raw[i][e]);
                    float d = Traits<T>::to_f32(grad[i][e]);
                    if (c.silu) {
                        const float pre = taps.pre(rows, e), g = sigmoid_of(pre);
                        d *= g * fmaf(pre, 1.0f - g, 1.0f);
                    }
                    if (!in) d = 0.0f;
#pragma unroll
                    for (int k = 0; k < W - 1; ++k) d_pre[k][e] = d_pre[k + 1][e];
                    d_pre[W - 1][e] = d;
                    float v = 0.0f;
#pragma unroll
                    for (int m = 0; m < W; ++m) v = fmaf(taps.w[W - 1 - m][e], d_pre[m][e], v);
                    out[e] = v;
                    if (own) {
                        d_b[e] += d;
#pragma unroll
                        for (int k = 0; k < W; ++k) d_w[k][e] = fmaf(d, rows[k][e], d_w[k][e]);
                    }
#pragma unroll
                    for (int k = 0; k < W - 1; ++k) rows[k][e] = rows[k + 1][e];
                }
                if (r < s.from && !(s.first && c.d_initial)) continue;
                const int left = r - (s.hi - (W - 1));      // row of the state behind the sequence
                if (c.d_final && left >= 0) {
                    float f[kVec];
                    load_row<T>((const T*)c.d_final + ((int64_t)s.sequence * (W - 1) + left) * c.channels, at, c.channels, f);
#pragma unroll
                    for (int e = 0; e < kVec; ++e) out[e] += f[e];
                }
                if (r >= s.from) store_row<T>(row_out<T>(c.d_x, r), at, c.channels, out);
                else store_row<T>((T*)c.d_initial + ((int64_t)s.sequence * (W - 1) + (r - s.lo + W - 1)) * c.channels, at, c.channels, out);
            }
        }
    }
    if (c.parts_at == nullptr) return;
    float* parts = c.parts_at + (int64_t)me.slot * c.channels * (W + 1);
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
        if (e < me.piece.skip || at + e >= c.channels) continue;
#pragma unroll
        for (int k = 0; k < W; ++k) parts[(int64_t)(at + e) * W + k] = d_w[k][e];
        parts[(int64_t)c.channels * W + at + e] = d_b[e];
    }
}

// One token for each sequence.  The state may be updated in place: where pieces share channels, each writes its own alone.
template <class T, int W>
__global__ void __launch_bounds__(256) conv_step_kernel(ConvCall c, int across, int blocks_across) {
    constexpr int kVec = Traits<T>::kVec;
    const Place<kVec> me(c.channels, across, blocks_across);
    if (!me.piece.live || me.slot >= c.slots.sequences) return;
    const int at = me.piece.at;
    const Taps<T, W> taps(c, at);
    float rows[W][kVec], out[kVec];
    const int64_t state = (int64_t)me.slot * (W - 1) * c.channels;
#pragma unroll
    for (int k = 0; k < W - 1; ++k) load_row<T>((const T*)c.initial + state + (int64_t)k * c.channels, at, c.channels, rows[k]);
    load_row<T>(row<T>(c.x, me.slot), at, c.channels, rows[W - 1]);
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
        const float pre = taps.pre(rows, e);
        out[e] = c.silu ? pre * sigmoid_of(pre) : pre;
    }
    if (me.piece.skip == 0) {
        store_row<T>(row_out<T>(c.out, me.slot), at, c.channels, out);
#pragma unroll
        for (int k = 0; k < W - 1; ++k) store_row<T>((T*)c.final_state + state + (int64_t)k * c.channels, at, c.channels, rows[k + 1]);
    } else {
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
            if (e < me.piece.skip) continue;
            row_out<T>(c.out, me.slot)[at + e] = Traits<T>::from_f32(out[e]);
#pragma unroll
            for (int k = 0; k < W - 1; ++k) ((T*)c.final_state)[state + (int64_t)k * c.channels + at + e] = Traits<T>::from_f32(rows[k + 1][e]);
        }
    }
}

template <class F>
hipError_t with_kind(int dt, int width, F&& f) {
    using std::integral_constant;
    auto of_width = [&](auto type) {
        switch (width) {
            case 2: return f(type, integral_constant<int, 2>{});
            case 3: return f(type, integral_constant<int, 3>{});
            case 4: return f(type, integral_constant<int, 4>{});
        }
        return hipErrorInvalidValue;
    };
    switch (dt) {
        case 0: return of_width(float{});
        case 1: return of_width(_Float16{});
        case 2: return of_width(__bf16{});
    }
    return hipErrorInvalidValue;
}

struct Grid { int across, blocks_across; };
Grid grid_of(int channels, int elem) {
    const int vec = 16 / elem, pieces = (channels + vec - 1) / vec;
    int across = 1;
    while (across < pieces && across < 256) across *= 2;
    return {across, (pieces + across - 1) / across};
}
unsigned blocks_of(const Grid& g, int64_t slots) { return (unsigned)((slots + 256 / g.across - 1) / (256 / g.across) * g.blocks_across); }

}  // namespace

hipError_t launch_conv_forward(int dt, const ConvCall& c, hipStream_t stream) {
    return with_kind(dt, c.width, [&](auto type, auto w) {
        typedef decltype(type) T;
        const Grid g = grid_of(c.channels, sizeof(T));
        const int64_t slots = slot_count(c.slots);
        hipLaunchKernelGGL((conv_kernel<T, decltype(w)::value>), dim3(blocks_of(g, slots)), dim3(256), 0, stream, c, g.across, g.blocks_across, (int)slots);
        return hipGetLastError();
    });
}

hipError_t launch_conv_backward(int dt, const ConvCall& c, hipStream_t stream) {
    return with_kind(dt, c.width, [&](auto type, auto w) {
        typedef decltype(type) T;
        const Grid g = grid_of(c.channels, sizeof(T));
        const int64_t slots = slot_count(c.slots), taps = (int64_t)c.channels * c.width;
        hipLaunchKernelGGL((conv_backward_kernel<T, decltype(w)::value>), dim3(blocks_of(g, slots)), dim3(256), 0, stream, c, g.across, g.blocks_across, (int)slots);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || c.parts_at == nullptr) return e;
        return launch_sum_parts(c.parts_at, slots, taps + c.channels, PartSums{{c.d_weight, c.d_bias, nullptr}, {taps, c.channels, 0}}, stream);
    });
}

hipError_t launch_conv_step(int dt, const ConvCall& c, hipStream_t stream) {
    return with_kind(dt, c.width, [&](auto type, auto w) {
        typedef decltype(type) T;
        const Grid g = grid_of(c.channels, sizeof(T));
        hipLaunchKernelGGL((conv_step_kernel<T, decltype(w)::value>), dim3(blocks_of(g, c.slots.sequences)), dim3(256), 0, stream, c, g.across, g.blocks_across);
        return hipGetLastError();
    });
}

}  // namespace msla
