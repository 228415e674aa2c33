// A scan whose states decay each at their own rate (selective state space):
//     t_i,c = softplus(delta_i,c + bias_c)        h_i[c, n] = exp(t_i,c a[c, n]) h_{i-1}[c, n] + t_i,c x_i,c b_i[n]
//     y_i,c = sum_n c_i[n] h_i[c, n] + skip_c x_i,c                out = y silu(gate)
// The decays differ for every channel and state, so no product of matrices is in it: a state and token is an exponential, two products and two
// multiply-adds on the vector units, and these bound it (the exponential costs two issue slots or more, the rest one each), not memory.
//
// Four lanes have a channel, a quarter of its states each (2 to 16) in registers: 16 channels a wave, 64 a workgroup.  Tokens go by in blocks of
// four: a lane loads and prepares one of them (step, gate), hands its step to the other three by data-parallel moves, and the four tokens' sums over
// states are exchanged so that each lane ends up with the one that it prepared, and stores it.
//
// Long sequences are cut into slots where channels alone do not fill the GPU: a pass over each slot from a state of zero, a join of the slots'
// states in their order (what a slot leaves of a state is exp(a * the sum of its steps)), then all slots from their own states.
//
// The gradient, with dh_i = c_i dy_i + exp(t_{i+1} a) dh_{i+1} and w_i = dh_i exp(t_i a) h_{i-1}:
//     d_c = sum over channels of dy h        d_b = sum over channels of dh t x        e = sum over n of dh b
//     d_t = x e + sum over n of w a          d_x = t e + skip dy                      d_a = sum over tokens of w t
// runs over the same slots.  The pass before the join sums exp(a * the steps up to i) c_i dy_i as well, which is what a slot adds to dh in front of
// it.  Then a slot goes through its tokens once to leave the state at every window of a few tokens in LDS, and through the windows from the end:
// states again, kept in registers, and back.  Sums over channels go over the lanes of a wave by exchanging halves (each step halves what a
// lane has), over the waves through LDS, over workgroups through parts in the workspace that a last launch adds up in a fixed order.
#include "msla_device.h"
#include "msla_layer_kernels.h"

namespace msla {
namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

__device__ __forceinline__ float exp2_of(float v) { return __builtin_amdgcn_exp2f(v); }
// (an exponential below fp32's normal range is zero, as its reciprocal's argument is then one)
__device__ __forceinline__ float sigmoid_of(float v) { return __builtin_amdgcn_rcpf(1.0f + exp2_of(-kLog2e * v)); }
// a in powers of two, finite: a rate of -infinity forgets everything in any step, and nothing in a step of 0
__device__ __forceinline__ float rate_of(float a) { return a < -2e38f ? -2e38f * kLog2e : a * kLog2e; }
// max(v, 0) + log(1 + e) with e = exp(-|v|): the logarithm of the rounded 1 + e, and what the rounding left out
__device__ __forceinline__ float softplus_of(float v) {
    const float e = exp2_of(-kLog2e * fabsf(v)), u = 1.0f + e;
    return fmaxf(v, 0.0f) + fmaf(__builtin_amdgcn_logf(u), kLn2, (e - (u - 1.0f)) * __builtin_amdgcn_rcpf(u));
}

template <int CTRL>
__device__ __forceinline__ float moved(float v) {
    const int b = __builtin_bit_cast(int, v);
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(b, b, CTRL, 0xf, 0xf, true));
}
// lane I of every four
template <int I>
__device__ __forceinline__ float of_four(float v) { return moved<I * 0x55>(v); }
// the sum over every four lanes of p[j], to lane j
__device__ __forceinline__ float deal_four(const float (&p)[4], bool odd, bool upper) {
    const float r0 = (odd ? p[1] : p[0]) + moved<0xB1>(odd ? p[0] : p[1]);      // (lane ^ 1)
    const float r1 = (odd ? p[3] : p[2]) + moved<0xB1>(odd ? p[2] : p[3]);
    return (upper ? r1 : r0) + moved<0x4E>(upper ? r0 : r1);                    // (lane ^ 2)
}
// lanes below 32 get a's sum over lane ^ 32, the others b's
__device__ __forceinline__ float halve32(float a, float b) {
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b), false, false);
    const unsigned first = r[0], second = r[1];        // (bit_cast of a vector's element itself reads element 0)
    return __builtin_bit_cast(float, first) + __builtin_bit_cast(float, second);
}
// even rows of 16 lanes get a's sum over lane ^ 16, odd ones b's
__device__ __forceinline__ float halve16(float a, float b) {
    const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b), false, false);
    const unsigned first = r[0], second = r[1];        // (bit_cast of a vector's element itself reads element 0)
    return __builtin_bit_cast(float, first) + __builtin_bit_cast(float, second);
}
// lanes without the 8 (the 4) get a's sum over lane ^ 8 (lane ^ 4), the others b's
__device__ __forceinline__ float halve8(float a, float b, bool mine_b) { return (mine_b ? b : a) + moved<0x128>(mine_b ? a : b); }
__device__ __forceinline__ float halve4(float a, float b, bool mine_b) {
    return (mine_b ? b : a) + moved<0x1B>(moved<0x141>(mine_b ? a : b));        // (7 - lane within eight, then 3 - lane within four)
}

// S neighbours of a row that starts anywhere
template <class T, int S>
struct Piece {
    T v[S];
    __device__ __forceinline__ void load(const T* p) { __builtin_memcpy(v, __builtin_assume_aligned(p, sizeof(T)), S * sizeof(T)); }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int s = 0; s < S; ++s) v[s] = Traits<T>::from_f32(0.0f);
    }
    __device__ __forceinline__ float at(int s) const { return Traits<T>::to_f32(v[s]); }
};

// What a lane is: its channel, its quarter of the states and its token of every four.
template <int S>
struct Place {
    int channel, group, quarter;
    bool live, odd, upper;
    __device__ __forceinline__ Place(const ScanCall& c, int tile) {
        const int per = c.channels / c.groups, tiles = (per + kScanTile - 1) / kScanTile;
        group = tile / tiles;
        const int at = tile % tiles * kScanTile + threadIdx.x / 4;
        live = at < per;
        channel = group * per + (live ? at : per - 1);
        quarter = threadIdx.x & 3;
        odd = threadIdx.x & 1;
        upper = threadIdx.x & 2;
    }
};

template <class T>
__device__ __forceinline__ const T* row(const TokenRows& r, int t) { return (const T*)r.p + (int64_t)t * r.ts; }
template <class T>
__device__ __forceinline__ T* row_out(const TokenRows& r, int t) { return (T*)r.p + (int64_t)t * r.ts; }

template <int S>
__device__ __forceinline__ void load_states(float (&to)[S], const float* p) { __builtin_memcpy(to, __builtin_assume_aligned(p, 4), S * 4); }
template <int S>
__device__ __forceinline__ void store_states(float* p, const float (&from)[S]) { __builtin_memcpy(__builtin_assume_aligned(p, 4), from, S * 4); }
// ... in LDS, where they lie on multiples of their own size
template <int S>
__device__ __forceinline__ void load_own(float (&to)[S], const float* p) { __builtin_memcpy(to, __builtin_assume_aligned(p, S >= 4 ? 16 : 8), S * 4); }
template <int S>
__device__ __forceinline__ void store_own(float* p, const float (&from)[S]) { __builtin_memcpy(__builtin_assume_aligned(p, S >= 4 ? 16 : 8), from, S * 4); }

enum Pass { kWhole, kSums, kSumsBoth };

// Four tokens as they are loaded: a lane's own, and its states' b and c of all four.
template <class T, int S, int PASS>
struct Block {
    T x, delta, gate, d_out;
    Piece<T, S> b[4], c[4];
};

// kWhole: outputs and the last state.  kSums: a slot's state from zero and the sum of its steps.  kSumsBoth: and what it adds to the gradient of the
// state in front of it.
template <class T, int S, int PASS>
__global__ void __launch_bounds__(kThreads) scan_kernel(ScanCall call, int tiles) {
    const Slot slot = slot_at(call.slots, blockIdx.x / tiles);
    if (!slot.used) return;
    const Place<S> me(call, blockIdx.x % tiles);
    constexpr int N = 4 * S;
    const int64_t state_at = (int64_t)me.channel * N + me.quarter * S, per_state = (int64_t)call.channels * N;
    const bool gated = call.gate.p != nullptr, soft = call.softplus != 0;
    float a[S], h[S];
    load_states(a, call.a + state_at);
#pragma unroll
    for (int s = 0; s < S; ++s) a[s] = rate_of(a[s]);
    const float bias = call.bias ? call.bias[me.channel] : 0.0f, skip = call.skip ? call.skip[me.channel] : 0.0f;
#pragma unroll
    for (int s = 0; s < S; ++s) h[s] = 0.0f;
    if constexpr (PASS == kWhole) {
        if (call.cut) load_states(h, call.states_at + (int64_t)(blockIdx.x / tiles) * per_state + state_at);
        else if (call.initial) load_states(h, call.initial + slot.sequence * per_state + state_at);
    }
    float along[S], reach[S];           // exp(a * the steps so far), and the sum of that times c dy
#pragma unroll
    for (int s = 0; s < S; ++s) along[s] = 1.0f, reach[s] = 0.0f;
    float steps = 0.0f;
    const int last = slot.until - 1;
    const int shared_at = me.group * N + me.quarter * S;
    typedef Block<T, S, PASS> B;
    auto fetch = [&](B& k, int t0) {
        if (t0 > last) return;
        const int t = min(t0 + me.quarter, last);
        k.x = row<T>(call.x, t)[me.channel];
        k.delta = row<T>(call.delta, t)[me.channel];
        if constexpr (PASS != kSums)
            if (gated) k.gate = row<T>(call.gate, t)[me.channel];
        if constexpr (PASS == kSumsBoth) k.d_out = row<T>(call.d_out, t)[me.channel];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int ti = min(t0 + i, last);
            k.b[i].load(row<T>(call.b, ti) + shared_at);
            if constexpr (PASS != kSums) k.c[i].load(row<T>(call.c, ti) + shared_at);
        }
    };
    auto advance = [&](B& k, int t0) {
        const bool in = t0 + me.quarter <= last;
        if (t0 + 3 > last) {            // (tokens behind the last one: a step of nothing, and nothing that is not finite)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (t0 + i > last) k.b[i].clear(), k.c[i].clear();
        }
        const float x = Traits<T>::to_f32(k.x), pre = Traits<T>::to_f32(k.delta) + bias;
        const float step = in ? (soft ? softplus_of(pre) : pre) : 0.0f, add = in ? step * x : 0.0f;
        float dy = 0.0f;
        if constexpr (PASS == kSumsBoth) {
            dy = Traits<T>::to_f32(k.d_out);
            if (gated) {
                const float z = Traits<T>::to_f32(k.gate);
                dy *= z * sigmoid_of(z);
            }
            if (!in) dy = 0.0f;
        }
        steps += step;
        float sums[4];
        auto token = [&](auto which) {
            constexpr int i = decltype(which)::value;
            const float ti = of_four<i>(step), ui = of_four<i>(add);
            float dyi = 0.0f;
            if constexpr (PASS == kSumsBoth) dyi = of_four<i>(dy);
            float y = 0.0f;
#pragma unroll
            for (int s = 0; s < S; ++s) {
                const float keep = exp2_of(ti * a[s]);
                h[s] = fmaf(keep, h[s], ui * k.b[i].at(s));
                if constexpr (PASS == kWhole) y = fmaf(k.c[i].at(s), h[s], y);
                if constexpr (PASS == kSumsBoth) {
                    along[s] *= keep;
                    reach[s] = fmaf(along[s] * dyi, k.c[i].at(s), reach[s]);
                }
            }
            sums[i] = y;
        };
        static_for<0, 4>(token);
        if constexpr (PASS == kWhole) {
            float y = fmaf(skip, x, deal_four(sums, me.odd, me.upper));
            if (gated) {
                const float z = Traits<T>::to_f32(k.gate);
                y *= z * sigmoid_of(z);
            }
            if (in && me.live) row_out<T>(call.out, t0 + me.quarter)[me.channel] = Traits<T>::from_f32(y);
        }
    };
    B here, there;
    fetch(here, slot.from);
    for (int t = slot.from; t <= last; t += 8) {
        fetch(there, t + 4);
        advance(here, t);
        if (t + 4 > last) break;
        fetch(here, t + 8);
        advance(there, t + 4);
    }
    if (!me.live) return;
    if constexpr (PASS == kWhole) {
        if (call.final_state && slot.last) store_states(call.final_state + slot.sequence * per_state + state_at, h);
    } else {
        const int64_t at = (int64_t)(blockIdx.x / tiles) * per_state + state_at;
        store_states(call.states_at + at, h);
        if constexpr (PASS == kSumsBoth) store_states(call.d_states_at + at, reach);
        // (a lane has the steps of its own tokens of every four)
        steps += moved<0xB1>(steps);
        steps += moved<0x4E>(steps);
        if (me.quarter == 0) call.steps_at[(int64_t)(blockIdx.x / tiles) * call.channels + me.channel] = steps;
    }
}

// The state that each slot starts from, and (BOTH) the state's gradient behind each slot, in the places of the slots' own sums.  A thread has one state
// of a sequence; the next slots' sums are on their way while one is joined.
template <bool BOTH>
__global__ void __launch_bounds__(256) scan_join_kernel(ScanCall call, int blocks) {
    const int b = blockIdx.x / blocks;
    const int64_t per_state = (int64_t)call.channels * call.states, at = (int64_t)(blockIdx.x % blocks) * 256 + threadIdx.x;
    if (at >= per_state) return;
    int lo, hi;
    rows_of_sequence(call.slots, b, lo, hi);
    // (a sequence without tokens has a slot, too, which hands its state on)
    const int64_t from = first_slot(call.slots, b), count = max(((int64_t)hi - lo + call.slots.run - 1) / call.slots.run, (int64_t)1);
    const float a = rate_of(call.a[at]);
    const int64_t channel = at / call.states;
    float h = call.initial ? call.initial[b * per_state + at] : 0.0f;
    constexpr int kAhead = 8;
    for (int64_t k0 = 0; k0 < count; k0 += kAhead) {
        float own[kAhead], steps[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int64_t slot = from + min(k0 + k, count - 1);
            own[k] = call.states_at[slot * per_state + at];
            steps[k] = call.steps_at[slot * call.channels + channel];
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (k0 + k < count) {
                call.states_at[(from + k0 + k) * per_state + at] = h;
                h = fmaf(exp2_of(a * steps[k]), h, own[k]);
            }
    }
    if constexpr (BOTH) {
        float g = call.d_final ? call.d_final[b * per_state + at] : 0.0f;
        for (int64_t k0 = 0; k0 < count; k0 += kAhead) {
            float own[kAhead], steps[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int64_t slot = from + max(count - 1 - k0 - k, (int64_t)0);
                own[k] = call.d_states_at[slot * per_state + at];
                steps[k] = call.steps_at[slot * call.channels + channel];
            }
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
                if (k0 + k < count) {
                    call.d_states_at[(from + count - 1 - k0 - k) * per_state + at] = g;
                    g = fmaf(exp2_of(a * steps[k]), g, own[k]);
                }
        }
    }
}

// A slot of the gradient.  K tokens a window, whose states stay in registers (K * S of them).
template <class T, int S>
struct Window {
    static constexpr int kTokens = S <= 4 ? 16 : 64 / S, kBlocks = kTokens / 4;
    T x[kBlocks], delta[kBlocks], gate[kBlocks], d_out[kBlocks];
};

template <class T, int S>
__global__ void __launch_bounds__(kThreads) scan_backward_kernel(ScanCall call, int tiles) {
    constexpr int N = 4 * S, K = Window<T, S>::kTokens, kBlocks = K / 4, kRun = N <= 32 ? 64 : 32, kWindows = kRun / K, kShared = K * 2 * N;
    // the states at the windows' starts, a lane's own; b and c of the slot in fp32; a window's sums over the channels of a wave
    __shared__ __align__(16) float marks[kWindows][kThreads * S];
    __shared__ __align__(16) float shared_bc[2][kRun * N];
    __shared__ float sums[2][kWaves][kShared];
    const int64_t slot_number = blockIdx.x / tiles;
    const int tile = blockIdx.x % tiles;
    const Slot slot = slot_at(call.slots, (int)slot_number);
    const Place<S> me(call, tile);
    const int64_t state_at = (int64_t)me.channel * N + me.quarter * S, per_state = (int64_t)call.channels * N;
    float* parts = call.parts_at + slot_number * (per_state + 2 * call.channels);
    float d_a[S], carry[S], h[S];
#pragma unroll
    for (int s = 0; s < S; ++s) d_a[s] = carry[s] = h[s] = 0.0f;
    float d_skip = 0.0f, d_bias = 0.0f;
    if (slot.used) {
        const bool gated = call.gate.p != nullptr, soft = call.softplus != 0;
        float a[S];
        load_states(a, call.a + state_at);
#pragma unroll
        for (int s = 0; s < S; ++s) a[s] = rate_of(a[s]);
        const float bias = call.bias ? call.bias[me.channel] : 0.0f, skip = call.skip ? call.skip[me.channel] : 0.0f;
        if (call.cut) {
            load_states(h, call.states_at + slot_number * per_state + state_at);
            load_states(carry, call.d_states_at + slot_number * per_state + state_at);
        } else {
            if (call.initial) load_states(h, call.initial + slot.sequence * per_state + state_at);
            if (call.d_final) load_states(carry, call.d_final + slot.sequence * per_state + state_at);
        }
        if (!me.live) {                 // (lanes without a channel read another's values, and must not add even an infinity to sums)
#pragma unroll
            for (int s = 0; s < S; ++s) carry[s] = h[s] = 0.0f;
        }
        const int count = slot.until - slot.from, last = slot.until - 1, windows = (count + K - 1) / K;
        for (int e = threadIdx.x; e < windows * K * N; e += kThreads) {
            const int t = e / N, n = e % N;
            const bool in = t < count;          // (zeros behind the last token)
            shared_bc[0][e] = in ? Traits<T>::to_f32(row<T>(call.b, slot.from + t)[me.group * N + n]) : 0.0f;
            shared_bc[1][e] = in ? Traits<T>::to_f32(row<T>(call.c, slot.from + t)[me.group * N + n]) : 0.0f;
        }
        __syncthreads();
        auto of_shared = [&](int which, int t) {
            struct { float v[S]; } r;
            load_own(r.v, &shared_bc[which][t * N + me.quarter * S]);
            return r;
        };
        // the state at each window's start
        for (int w = 0; w < windows; ++w) {
            store_own(&marks[w][threadIdx.x * S], h);
            if (w + 1 == windows) break;
            float step[kBlocks], add[kBlocks];
#pragma unroll
            for (int q = 0; q < kBlocks; ++q) {
                const int t = min(slot.from + w * K + 4 * q + me.quarter, last);
                const float pre = Traits<T>::to_f32(row<T>(call.delta, t)[me.channel]) + bias;
                step[q] = soft ? softplus_of(pre) : pre;
                add[q] = step[q] * Traits<T>::to_f32(row<T>(call.x, t)[me.channel]);
            }
            static_for<0, K>([&](auto which) {
                constexpr int t = decltype(which)::value, q = t / 4, i = t % 4;
                const auto b = of_shared(0, w * K + t);
                const float ti = of_four<i>(step[q]), ui = of_four<i>(add[q]);
#pragma unroll
                for (int s = 0; s < S; ++s) h[s] = fmaf(exp2_of(ti * a[s]), h[s], ui * b.v[s]);
            });
        }
        Window<T, S> now, next;
        auto fetch = [&](Window<T, S>& to, int w) {
#pragma unroll
            for (int q = 0; q < kBlocks; ++q) {
                const int t = min(slot.from + w * K + 4 * q + me.quarter, last);
                to.x[q] = row<T>(call.x, t)[me.channel];
                to.delta[q] = row<T>(call.delta, t)[me.channel];
                to.d_out[q] = row<T>(call.d_out, t)[me.channel];
                if (gated) to.gate[q] = row<T>(call.gate, t)[me.channel];
            }
        };
        if (windows > 0) fetch(now, windows - 1);
        for (int w = windows - 1; w >= 0; --w) {
            if (w > 0) fetch(next, w - 1);
            float step[kBlocks], add[kBlocks], dy[kBlocks];
#pragma unroll
            for (int q = 0; q < kBlocks; ++q) {
                const bool in = w * K + 4 * q + me.quarter < count && me.live;
                const float pre = Traits<T>::to_f32(now.delta[q]) + bias, x = Traits<T>::to_f32(now.x[q]);
                step[q] = in ? (soft ? softplus_of(pre) : pre) : 0.0f;
                add[q] = in ? step[q] * x : 0.0f;
                dy[q] = in ? Traits<T>::to_f32(now.d_out[q]) : 0.0f;
            }
            float states[K][S];             // behind each token
            load_own(h, &marks[w][threadIdx.x * S]);
            float before[S];
#pragma unroll
            for (int s = 0; s < S; ++s) before[s] = h[s];
            static_for<0, kBlocks>([&](auto block) {
                constexpr int q = decltype(block)::value;
                float y4[4];
                static_for<0, 4>([&](auto which) {
                    constexpr int i = decltype(which)::value, t = 4 * q + i;
                    const auto b = of_shared(0, w * K + t);
                    const float ti = of_four<i>(step[q]), ui = of_four<i>(add[q]);
#pragma unroll
                    for (int s = 0; s < S; ++s) states[t][s] = h[s] = fmaf(exp2_of(ti * a[s]), h[s], ui * b.v[s]);
                    y4[i] = 0.0f;
                    if (gated) {
                        const auto c = of_shared(1, w * K + t);
#pragma unroll
                        for (int s = 0; s < S; ++s) y4[i] = fmaf(c.v[s], h[s], y4[i]);
                    }
                });
                if (gated) {
                    const float z = Traits<T>::to_f32(now.gate[q]), x = Traits<T>::to_f32(now.x[q]);
                    const float y = fmaf(skip, x, deal_four(y4, me.odd, me.upper)), g = sigmoid_of(z);
                    const int t = w * K + 4 * q + me.quarter;
                    if (t < count && me.live)
                        row_out<T>(call.d_gate, slot.from + t)[me.channel] = Traits<T>::from_f32(dy[q] * y * (g * fmaf(z, 1.0f - g, 1.0f)));
                    dy[q] = t < count && me.live ? dy[q] * (z * g) : 0.0f;
                }
            });
            float(&room)[kWaves][kShared] = sums[w & 1];
            static_for<0, kBlocks>([&](auto back) {
                constexpr int q = kBlocks - 1 - decltype(back)::value;
                float e4[4], w4[4], both[4][S / 2];
                static_for<0, 4>([&](auto behind) {
                    constexpr int i = 3 - decltype(behind)::value, t = 4 * q + i;
                    const auto b = of_shared(0, w * K + t), c = of_shared(1, w * K + t);
                    const float ti = of_four<i>(step[q]), ui = of_four<i>(add[q]), dyi = of_four<i>(dy[q]);
                    float e = 0.0f, along = 0.0f, r[S];
#pragma unroll
                    for (int s = 0; s < S; ++s) {
                        const float dh = fmaf(c.v[s], dyi, carry[s]);
                        r[s] = halve32(dh * ui, dyi * states[t][s]);
                        e = fmaf(dh, b.v[s], e);
                        carry[s] = exp2_of(ti * a[s]) * dh;
                        const float through = carry[s] * (t > 0 ? states[t > 0 ? t - 1 : 0][s] : before[s]);
                        d_a[s] = fmaf(through, ti, d_a[s]);
                        along = fmaf(through, a[s], along);
                    }
#pragma unroll
                    for (int p = 0; p < S / 2; ++p) both[i][p] = halve16(r[2 * p], r[2 * p + 1]);
                    e4[i] = e;
                    w4[i] = along;
                });
                // sums over the channels of the wave: a lane ends up with those of b or c (its 32), an odd or even state (its 16), one token of the
                // four (its 8 and 4)
                const int lane = threadIdx.x & 63;
                const bool mine8 = lane & 8, mine4 = lane & 4;
#pragma unroll
                for (int p = 0; p < S / 2; ++p) {
                    const float lower = halve8(both[0][p], both[2][p], mine8), higher = halve8(both[1][p], both[3][p], mine8);
                    const float v = halve4(lower, higher, mine4);
                    const int token = 4 * q + (mine8 ? 2 : 0) + (mine4 ? 1 : 0);
                    room[threadIdx.x >> 6][token * 2 * N + (lane & 32 ? N : 0) + me.quarter * S + 2 * p + (lane & 16 ? 1 : 0)] = v;
                }
                const float e = deal_four(e4, me.odd, me.upper), along = kLn2 * deal_four(w4, me.odd, me.upper);
                const float x = Traits<T>::to_f32(now.x[q]);
                const int t = w * K + 4 * q + me.quarter;
                float d_step = fmaf(x, e, along);
                if (soft) d_step *= sigmoid_of(Traits<T>::to_f32(now.delta[q]) + bias);
                if (t < count && me.live) {
                    row_out<T>(call.d_x, slot.from + t)[me.channel] = Traits<T>::from_f32(fmaf(step[q], e, skip * dy[q]));
                    row_out<T>(call.d_delta, slot.from + t)[me.channel] = Traits<T>::from_f32(d_step);
                    d_skip = fmaf(dy[q], x, d_skip);
                    d_bias += d_step;
                }
            });
            __syncthreads();
            // (one barrier a window: the room that the next one fills was last read before this one)
            const int tokens = min(K, count - w * K);
            for (int e = threadIdx.x; e < tokens * 2 * N; e += kThreads) {
                float v = room[0][e];
#pragma unroll
                for (int k = 1; k < kWaves; ++k) v += room[k][e];
                call.shared_at[((int64_t)tile * call.slots.tokens + slot.from + w * K) * (2 * N) + e] = v;
            }
            now = next;
        }
        if (slot.first && call.d_initial && me.live) store_states(call.d_initial + slot.sequence * per_state + state_at, carry);
    }
    d_skip += moved<0xB1>(d_skip);
    d_skip += moved<0x4E>(d_skip);
    d_bias += moved<0xB1>(d_bias);
    d_bias += moved<0x4E>(d_bias);
    if (!me.live) return;
    store_states(parts + state_at, d_a);
    if (me.quarter == 0) {
        parts[per_state + me.channel] = d_skip;
        parts[per_state + call.channels + me.channel] = d_bias;
    }
}

// d_b and d_c: sums over the tiles of a group.  A thread has one state of one token.
template <class T>
__global__ void __launch_bounds__(256) scan_shared_kernel(ScanCall call, int tiles) {
    const int n = call.states, per_row = call.groups * n;
    const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x, t = e / (2 * per_row);
    if (t >= call.slots.tokens) return;
    if (call.slots.offsets) {           // (rows of no sequence are left as they are)
        const int lo = call.slots.offsets[0], hi = call.slots.offsets[call.slots.sequences];
        if (t < lo || t >= hi) return;
    }
    const int at = (int)(e % (2 * per_row)), group = at / (2 * n), k = at % (2 * n), per_group = tiles / call.groups;
    float s = 0.0f;
#pragma unroll 8
    for (int i = 0; i < per_group; ++i) s += call.shared_at[((int64_t)(group * per_group + i) * call.slots.tokens + t) * (2 * n) + k];
    const TokenRows& to = k < n ? call.d_b : call.d_c;
    row_out<T>(to, (int)t)[group * n + k % n] = Traits<T>::from_f32(s);
}

// One token for each sequence: bound by the states, which are read and written once, 16 bytes a lane and access (16 states).
template <class T, int S>
__global__ void __launch_bounds__(256) scan_step_kernel(ScanCall call, int blocks) {
    constexpr int N = 4 * S;
    const int b = blockIdx.x / blocks, at = blockIdx.x % blocks * 64 + threadIdx.x / 4, quarter = threadIdx.x & 3;
    const bool live = at < call.channels;
    const int channel = live ? at : call.channels - 1, group = channel / (call.channels / call.groups);
    const int64_t place = ((int64_t)b * call.channels + channel) * N + quarter * S;
    float h[S], a[S];
    load_states(h, call.initial + place);
    load_states(a, call.a + (int64_t)channel * N + quarter * S);
    Piece<T, S> kb, kc;
    kb.load(row<T>(call.b, b) + group * N + quarter * S);
    kc.load(row<T>(call.c, b) + group * N + quarter * S);
    const float x = Traits<T>::to_f32(row<T>(call.x, b)[channel]), pre = Traits<T>::to_f32(row<T>(call.delta, b)[channel]) + (call.bias ? call.bias[channel] : 0.0f);
    const float step = call.softplus ? softplus_of(pre) : pre;
    float y = 0.0f;
#pragma unroll
    for (int s = 0; s < S; ++s) {
        h[s] = fmaf(exp2_of(step * rate_of(a[s])), h[s], step * x * kb.at(s));
        y = fmaf(kc.at(s), h[s], y);
    }
    y += moved<0xB1>(y);
    y += moved<0x4E>(y);
    if (!live) return;
    store_states(call.final_state + place, h);
    if (quarter != 0) return;
    if (call.skip) y = fmaf(call.skip[channel], x, y);
    if (call.gate.p) {
        const float z = Traits<T>::to_f32(row<T>(call.gate, b)[channel]);
        y *= z * sigmoid_of(z);
    }
    row_out<T>(call.out, b)[channel] = Traits<T>::from_f32(y);
}

template <class F>
hipError_t with_states(int states, F&& f) {
    using std::integral_constant;
    switch (states) {
        case 8: return f(integral_constant<int, 2>{});
        case 16: return f(integral_constant<int, 4>{});
        case 32: return f(integral_constant<int, 8>{});
        case 64: return f(integral_constant<int, 16>{});
    }
    return hipErrorInvalidValue;
}
template <class F>
hipError_t with_type(int dt, F&& f) {
    switch (dt) {
        case 0: return f(float{});
        case 1: return f(_Float16{});
        case 2: return f(__bf16{});
    }
    return hipErrorInvalidValue;
}

template <bool BOTH>
hipError_t join(const ScanCall& c, hipStream_t stream) {
    const int blocks = (int)(((int64_t)c.channels * c.states + 255) / 256);
    hipLaunchKernelGGL((scan_join_kernel<BOTH>), dim3((unsigned)blocks * (unsigned)c.slots.sequences), dim3(256), 0, stream, c, blocks);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_scan_forward(int dt, const ScanCall& c, hipStream_t stream) {
    return with_type(dt, [&](auto type) {
        typedef decltype(type) T;
        return with_states(c.states, [&](auto s) {
            constexpr int S = decltype(s)::value;
            const int tiles = scan_tiles(c.channels, c.groups);
            const dim3 grid((unsigned)(slot_count(c.slots) * tiles)), threads(kThreads);
            if (c.cut) {
                hipLaunchKernelGGL((scan_kernel<T, S, kSums>), grid, threads, 0, stream, c, tiles);
                hipError_t e = hipGetLastError();
                if (e == hipSuccess) e = join<false>(c, stream);
                if (e != hipSuccess) return e;
            }
            hipLaunchKernelGGL((scan_kernel<T, S, kWhole>), grid, threads, 0, stream, c, tiles);
            return hipGetLastError();
        });
    });
}

hipError_t launch_scan_backward(int dt, const ScanCall& c, hipStream_t stream) {
    return with_type(dt, [&](auto type) {
        typedef decltype(type) T;
        return with_states(c.states, [&](auto s) {
            constexpr int S = decltype(s)::value;
            const int tiles = scan_tiles(c.channels, c.groups);
            const int64_t slots = slot_count(c.slots);
            const dim3 grid((unsigned)(slots * tiles)), threads(kThreads);
            hipError_t e = hipSuccess;
            if (c.cut) {
                hipLaunchKernelGGL((scan_kernel<T, S, kSumsBoth>), grid, threads, 0, stream, c, tiles);
                e = hipGetLastError();
                if (e == hipSuccess) e = join<true>(c, stream);
                if (e != hipSuccess) return e;
            }
            hipLaunchKernelGGL((scan_backward_kernel<T, S>), grid, threads, 0, stream, c, tiles);
            e = hipGetLastError();
            if (e != hipSuccess) return e;
            const int64_t shared = (int64_t)c.slots.tokens * c.groups * c.states * 2;
            if (shared > 0) {
                hipLaunchKernelGGL((scan_shared_kernel<T>), dim3((unsigned)((shared + 255) / 256)), dim3(256), 0, stream, c, tiles);
                e = hipGetLastError();
                if (e != hipSuccess) return e;
            }
            const int64_t per_state = (int64_t)c.channels * c.states;
            return launch_sum_parts(c.parts_at, slots, per_state + 2 * c.channels,
                                    PartSums{{c.d_a, c.d_skip, c.d_bias}, {per_state, c.channels, c.channels}}, stream);
        });
    });
}

hipError_t launch_scan_step(int dt, const ScanCall& c, hipStream_t stream) {
    return with_type(dt, [&](auto type) {
        typedef decltype(type) T;
        return with_states(c.states, [&](auto s) {
            constexpr int S = decltype(s)::value;
            const int blocks = (c.channels + 63) / 64;
            hipLaunchKernelGGL((scan_step_kernel<T, S>), dim3((unsigned)(blocks * c.slots.sequences)), dim3(256), 0, stream, c, blocks);
            return hipGetLastError();
        });
    });
}

}  // namespace msla
