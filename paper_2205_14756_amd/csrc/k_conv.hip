// The short causal convolution of each channel with its own taps, over sequences: pre_i = bias + sum_k w[k] x_{i - width + 1 + k}, out = pre or silu(pre).
//
// Bound by memory.  A thread has a piece of 8 bytes of the channels and a run of tokens of one sequence (a slot), whose last width - 1 rows stay in registers as the
// run goes on; those before the run are read once more (out of a cache).  The sequence's state is those rows: the ones in front of its first
// token, and the last ones.  16384 tokens of 4096 channels in bf16, width 4: 63 us, 4.3 TB/s.
//
// The gradient goes over the same runs and the width - 1 tokens behind them, whose part of d_x it needs: pre again, d_pre = d_out silu'(pre), d_x_i = sum_m
// w[width - 1 - m] d_pre_{i + m}; taps and bias are summed over a run in registers, over runs through parts that a second launch adds up.  The same rows: 114 us
// and 6 for the parts, 3.4 TB/s at the three waves a SIMD that its 161 registers leave.  (Three in fp16 as well; two of width 3 in bf16, which takes 170; four of the others.)
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

// VEC neighbours of a row that starts anywhere
template <class T, int VEC>
struct Raw {
    T v[VEC];
    __device__ __forceinline__ void load(const T* p) { __builtin_memcpy(v, __builtin_assume_aligned(p, sizeof(T)), VEC * sizeof(T)); }
    __device__ __forceinline__ void store(T* p) const { __builtin_memcpy(__builtin_assume_aligned(p, sizeof(T)), v, VEC * sizeof(T)); }
    __device__ __forceinline__ float at(int e) const { return Traits<T>::to_f32(v[e]); }
    __device__ __forceinline__ void set(int e, float f) { v[e] = Traits<T>::from_f32(f); }
};

// A thread's place: `across` lanes (a power of two, 256 at most) take neighbouring pieces of a row, so that a wave reads whole lines.
template <int VEC>
struct Place {
    Piece<VEC> piece;
    int slot;
    __device__ __forceinline__ Place(int channels, int across, int blocks_across)
        : piece((int)(blockIdx.x % blocks_across) * across + (int)(threadIdx.x % across), channels),
          slot((int)(blockIdx.x / blocks_across) * (256 / across) + (int)(threadIdx.x / across)) {}
};

template <class T, int W, int VEC>
struct Taps {
    float w[W][VEC], bias[VEC];
    __device__ __forceinline__ Taps(const ConvCall& c, int at) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
#pragma unroll
            for (int k = 0; k < W; ++k) w[k][e] = Traits<T>::to_f32(((const T*)c.weight)[(int64_t)(at + e) * W + k]);
            bias[e] = c.bias ? Traits<T>::to_f32(((const T*)c.bias)[at + e]) : 0.0f;
        }
    }
    // of the token in rows[i + W - 1]
    template <int N>
    __device__ __forceinline__ float pre(const float (&rows)[N][VEC], int i, int e) const {
        float v = bias[e];
#pragma unroll
        for (int k = 0; k < W; ++k) v = fmaf(w[k][e], rows[i + k][e], v);
        return v;
    }
};

// the width - 1 rows in front of token t of a sequence that starts at lo, oldest first, to rows[0 .. W - 2]
template <class T, int W, int VEC, int N>
__device__ __forceinline__ void rows_before(const ConvCall& c, const Slot& s, int t, int at, float (&rows)[N][VEC]) {
#pragma unroll
    for (int k = 0; k < W - 1; ++k) {
        const int i = t - (W - 1) + k;
        Raw<T, VEC> r = {};
        if (i >= s.lo) r.load(row<T>(c.x, i) + at);
        else if (c.initial) r.load((const T*)c.initial + ((int64_t)s.sequence * (W - 1) + (W - 1 - (s.lo - i))) * c.channels + at);
#pragma unroll
        for (int e = 0; e < VEC; ++e) rows[k][e] = r.at(e);
    }
}

constexpr int kAhead = 4;       // tokens of a step: they are asked for a step ahead, and without a branch, so that a step waits for its own alone

template <class T, int W, int VEC>
__global__ void __launch_bounds__(256) conv_kernel(ConvCall c, int across, int blocks_across, int slots) {
    const Place<VEC> me(c.channels, across, blocks_across);
    if (!me.piece.live || me.slot >= slots) return;
    const Slot s = slot_at(c.slots, me.slot);
    if (!s.used) return;
    const int at = me.piece.at;
    Raw<T, VEC> next[kAhead];
    auto fetch = [&](int t0) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) next[i].load(row<T>(c.x, min(t0 + i, s.until - 1)) + at);
    };
    if (s.from < s.until) fetch(s.from);
    const Taps<T, W, VEC> taps(c, at);
    float rows[W - 1 + kAhead][VEC];
    rows_before<T, W, VEC>(c, s, s.from, at, rows);
    auto output = [&](int i) {
        Raw<T, VEC> out;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const float pre = taps.pre(rows, i, e), open = pre * sigmoid_of(pre);
            out.set(e, c.silu ? open : pre);
        }
        return out;
    };
    int t0 = s.from;
    for (; t0 + kAhead <= s.until; t0 += kAhead) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
#pragma unroll
            for (int e = 0; e < VEC; ++e) rows[W - 1 + i][e] = next[i].at(e);
        fetch(t0 + kAhead);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) output(i).store(row_out<T>(c.out, t0 + i) + at);
#pragma unroll
        for (int k = 0; k < W - 1; ++k)
#pragma unroll
            for (int e = 0; e < VEC; ++e) rows[k][e] = rows[k + kAhead][e];
    }
#pragma unroll
    for (int i = 0; i < kAhead - 1; ++i) {
        if (t0 + i >= s.until) break;
#pragma unroll
        for (int e = 0; e < VEC; ++e) rows[W - 1][e] = next[i].at(e);
        output(0).store(row_out<T>(c.out, t0 + i) + at);
#pragma unroll
        for (int k = 0; k < W - 1; ++k)
#pragma unroll
            for (int e = 0; e < VEC; ++e) rows[k][e] = rows[k + 1][e];
    }
    if (s.last && c.final_state) {
#pragma unroll
        for (int k = 0; k < W - 1; ++k) {
            Raw<T, VEC> out;
#pragma unroll
            for (int e = 0; e < VEC; ++e) out.set(e, rows[k][e]);
            out.store((T*)c.final_state + ((int64_t)s.sequence * (W - 1) + k) * c.channels + at);
        }
    }
}

template <class T, int W, int VEC>
__global__ void __launch_bounds__(256) conv_backward_kernel(ConvCall c, int across, int blocks_across, int slots) {
    const Place<VEC> me(c.channels, across, blocks_across);
    if (!me.piece.live || me.slot >= slots) return;
    const Slot s = slot_at(c.slots, me.slot);
    const int at = me.piece.at;
    float d_w[W][VEC], d_b[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
        d_b[e] = 0.0f;
#pragma unroll
        for (int k = 0; k < W; ++k) d_w[k][e] = 0.0f;
    }
    if (s.used) {
        Raw<T, VEC> next_x[kAhead], next_g[kAhead];
        auto fetch = [&](int t0) {
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int t = min(t0 + i, s.hi - 1);
                next_x[i].load(row<T>(c.x, t) + at);
                next_g[i].load(row<T>(c.d_out, t) + at);
            }
        };
        // the tokens whose outputs, width - 1 tokens back, are the run's own and know nothing of the state behind the sequence: whole steps of them
        const int steady = s.from + W - 1, steps = max(0, s.until - steady) / kAhead;
        if (steps > 0) fetch(steady);
        const Taps<T, W, VEC> taps(c, at);
        float rows[W - 1 + kAhead][VEC], d_pre[W - 1 + kAhead][VEC];        // of the last W - 1 tokens, and a step's
        rows_before<T, W, VEC>(c, s, s.from, at, rows);
#pragma unroll
        for (int k = 0; k < W - 1; ++k)
#pragma unroll
            for (int e = 0; e < VEC; ++e) d_pre[k][e] = 0.0f;
        // the token in rows[i + W - 1], whose output's gradient is g: d_pre of it, its part of the taps' gradient
        auto take = [&](int i, const Raw<T, VEC>& g, bool own, bool in) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const float pre = taps.pre(rows, i, e), open = sigmoid_of(pre), slope = open * fmaf(pre, 1.0f - open, 1.0f), back = g.at(e);
                const float d = in ? (c.silu ? back * slope : back) : 0.0f;
                d_pre[W - 1 + i][e] = d;
                if (own) {
                    d_b[e] += d;
#pragma unroll
                    for (int k = 0; k < W; ++k) d_w[k][e] = fmaf(d, rows[i + k][e], d_w[k][e]);
                }
            }
        };
        // d_x of the token W - 1 in front of that one
        auto give = [&](int i, float (&out)[VEC]) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                float v = 0.0f;
#pragma unroll
                for (int m = 0; m < W; ++m) v = fmaf(taps.w[W - 1 - m][e], d_pre[i + m][e], v);
                out[e] = v;
            }
        };
        auto shift = [&](int by) {
#pragma unroll
            for (int k = 0; k < W - 1; ++k)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    rows[k][e] = rows[k + by][e];
                    d_pre[k][e] = d_pre[k + by][e];
                }
        };
        auto edge = [&](int t) {
            const bool own = t < s.until, in = t < s.hi;
            const int r = t - (W - 1);
            Raw<T, VEC> x = {}, g = {};
            if (in) {
                x.load(row<T>(c.x, t) + at);
                g.load(row<T>(c.d_out, t) + at);
            }
#pragma unroll
            for (int e = 0; e < VEC; ++e) rows[W - 1][e] = x.at(e);
            take(0, g, own, in);
            float out[VEC];
            give(0, out);
            shift(1);
            if (r < s.from && !(s.first && c.d_initial)) return;
            const int left = r - (s.hi - (W - 1));      // row of the state behind the sequence
            if (c.d_final && left >= 0) {
                Raw<T, VEC> f;
                f.load((const T*)c.d_final + ((int64_t)s.sequence * (W - 1) + left) * c.channels + at);
#pragma unroll
                for (int e = 0; e < VEC; ++e) out[e] += f.at(e);
            }
            Raw<T, VEC> to;
#pragma unroll
            for (int e = 0; e < VEC; ++e) to.set(e, out[e]);
            to.store((r >= s.from ? row_out<T>(c.d_x, r) : (T*)c.d_initial + ((int64_t)s.sequence * (W - 1) + (r - s.lo + W - 1)) * c.channels) + at);
        };
        const int beyond = s.until + W - 1, first_edge = min(steady, beyond);
#pragma unroll 1
        for (int t = s.from; t < first_edge; ++t) edge(t);
        for (int n = 0; n < steps; ++n) {
            const int t0 = steady + n * kAhead;
            Raw<T, VEC> g[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                g[i] = next_g[i];
#pragma unroll
                for (int e = 0; e < VEC; ++e) rows[W - 1 + i][e] = next_x[i].at(e);
            }
            fetch(t0 + kAhead);
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                take(i, g[i], true, true);
                float out[VEC];
                give(i, out);
                Raw<T, VEC> to;
#pragma unroll
                for (int e = 0; e < VEC; ++e) to.set(e, out[e]);
                to.store(row_out<T>(c.d_x, t0 + i - (W - 1)) + at);
            }
            shift(kAhead);
        }
#pragma unroll 1
        for (int t = first_edge + steps * kAhead; t < beyond; ++t) edge(t);
    }
    if (c.parts_at == nullptr) return;
    float* parts = c.parts_at + (int64_t)me.slot * c.channels * (W + 1);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
        if (e < me.piece.skip) continue;
#pragma unroll
        for (int k = 0; k < W; ++k) parts[(int64_t)(at + e) * W + k] = d_w[k][e];
        parts[(int64_t)c.channels * W + at + e] = d_b[e];
    }
}

// One token for each sequence.  The state may be updated in place: where pieces share channels, each writes its own alone.
template <class T, int W, int VEC>
__global__ void __launch_bounds__(256) conv_step_kernel(ConvCall c, int across, int blocks_across) {
    const Place<VEC> me(c.channels, across, blocks_across);
    if (!me.piece.live || me.slot >= c.slots.sequences) return;
    const int at = me.piece.at;
    const Taps<T, W, VEC> taps(c, at);
    const int64_t state = (int64_t)me.slot * (W - 1) * c.channels + at;
    Raw<T, VEC> raw[W], out;
    float rows[W][VEC];
#pragma unroll
    for (int k = 0; k < W - 1; ++k) raw[k].load((const T*)c.initial + state + (int64_t)k * c.channels);
    raw[W - 1].load(row<T>(c.x, me.slot) + at);
#pragma unroll
    for (int k = 0; k < W; ++k)
#pragma unroll
        for (int e = 0; e < VEC; ++e) rows[k][e] = raw[k].at(e);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
        const float pre = taps.pre(rows, 0, e), open = pre * sigmoid_of(pre);
        out.set(e, c.silu ? open : pre);
    }
    T* to = row_out<T>(c.out, me.slot) + at;
    T* states = (T*)c.final_state + state;
    if (me.piece.skip == 0) {
        out.store(to);
#pragma unroll
        for (int k = 0; k < W - 1; ++k) raw[k + 1].store(states + (int64_t)k * c.channels);
    } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            if (e < me.piece.skip) continue;
            to[e] = out.v[e];
#pragma unroll
            for (int k = 0; k < W - 1; ++k) states[(int64_t)k * c.channels + e] = raw[k + 1].v[e];
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

// Pieces of 8 bytes (what a lane keeps for each of its channels, taps and rows, in the gradient those of both, leaves 16-byte ones two or three waves a
// SIMD); of one element where a row is no longer than that.
template <class T, class F>
hipError_t with_pieces(int channels, F&& f) {
    constexpr int kVec = 8 / sizeof(T);
    auto launch = [&](auto vec) {
        const int pieces = (channels + decltype(vec)::value - 1) / decltype(vec)::value;
        int across = 1;
        while (across < pieces && across < 256) across *= 2;
        const int blocks_across = (pieces + across - 1) / across;
        f(vec, across, blocks_across, [=](int64_t slots) { return dim3((unsigned)((slots + 256 / across - 1) / (256 / across) * blocks_across)); });
        return hipGetLastError();
    };
    if (channels >= kVec) return launch(std::integral_constant<int, kVec>{});
    return launch(std::integral_constant<int, 1>{});
}

}  // namespace

hipError_t launch_conv_forward(int dt, const ConvCall& c, hipStream_t stream) {
    return with_kind(dt, c.width, [&](auto type, auto w) {
        typedef decltype(type) T;
        return with_pieces<T>(c.channels, [&](auto vec, int across, int blocks_across, auto grid) {
            const int64_t slots = slot_count(c.slots);
            hipLaunchKernelGGL((conv_kernel<T, decltype(w)::value, decltype(vec)::value>), grid(slots), dim3(256), 0, stream, c, across, blocks_across, (int)slots);
        });
    });
}

hipError_t launch_conv_backward(int dt, const ConvCall& c, hipStream_t stream) {
    return with_kind(dt, c.width, [&](auto type, auto w) {
        typedef decltype(type) T;
        const int64_t slots = slot_count(c.slots), taps = (int64_t)c.channels * c.width;
        const hipError_t e = with_pieces<T>(c.channels, [&](auto vec, int across, int blocks_across, auto grid) {
            hipLaunchKernelGGL((conv_backward_kernel<T, decltype(w)::value, decltype(vec)::value>), grid(slots), dim3(256), 0, stream, c, across, blocks_across, (int)slots);
        });
        if (e != hipSuccess || c.parts_at == nullptr) return e;
        return launch_sum_parts(c.parts_at, slots, taps + c.channels, PartSums{{c.d_weight, c.d_bias, nullptr}, {taps, c.channels, 0}}, stream);
    });
}

hipError_t launch_conv_step(int dt, const ConvCall& c, hipStream_t stream) {
    return with_kind(dt, c.width, [&](auto type, auto w) {
        typedef decltype(type) T;
        return with_pieces<T>(c.channels, [&](auto vec, int across, int blocks_across, auto grid) {
            hipLaunchKernelGGL((conv_step_kernel<T, decltype(w)::value, decltype(vec)::value>), grid(c.slots.sequences), dim3(256), 0, stream, c, across, blocks_across);
        });
    });
}

}  // namespace msla
