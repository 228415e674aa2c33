// A scan whose states decay each at their own rate (selective state space):
//     t_i,c = softplus(delta_i,c + bias_c)        h_i[c, n] = exp(t_i,c a[c, n]) h_{i-1}[c, n] + t_i,c x_i,c b_i[n]
//     y_i,c = sum_n c_i[n] h_i[c, n] + skip_c x_i,c                out = y silu(gate)
// The decays differ for every channel and state, so no product of matrices is in it: a state and token is an exponential, two products and two
// multiply-adds on the vector units, and their issue bounds it (the exponential costs two slots), not memory.  8192 tokens of 4096 channels of 16 states in bf16: 172 us,
// 1.6 TB/s; the vector units are busy for 0.9 of the cycles, with 9.6 instructions a state and token, 5 of them the recurrence's own.
//
// Sixteen lanes have a channel (eight where it has 8 states) and its states in registers.  Sums over the states of as many tokens as there are lanes are exchanged so that
// each lane ends up with one token's.  Sequences are cut into slots where channels alone do not fill the GPU: a pass over each slot from a state of zero, a join
// of the slots' states in their order (what a slot leaves of a state is exp(a * the sum of its steps)), then all slots from their own states.
//
// The gradient, with dh_i = c_i dy_i + exp(t_{i+1} a) dh_{i+1} and w_i = dh_i exp(t_i a) h_{i-1}:
//     d_c = sum over channels of dy h        d_b = sum over channels of dh t x        e = sum over n of dh b
//     d_t = x e + sum over n of w a          d_x = t e + skip dy                      d_a = sum over tokens of w t
// runs over slots as well.  A pass forward leaves the state at every 16 tokens (a mark); where sequences are cut it also sums exp(a * the steps up to i) c_i dy_i, which is
// what a slot adds to dh in front of it.  The pass back makes 16 tokens' states again from their mark, keeps them in registers, and goes back over them.  Sums
// over channels go over the lanes of a wave by exchanging halves, over the waves through LDS, over workgroups through parts in the workspace that a last
// launch adds up in a fixed order.  The same tokens and channels: 751 us, of which the pass back 597 (vector units busy for 0.75 of the cycles, 29 instructions a state and token).
#include "msla_device.h"
#include "msla_layer_kernels.h"
#include "scan_lanes.h"

namespace msla {
namespace {

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

// What a lane is: its channel, and its number among the L that share it.  A workgroup has kScanSlice of them, of one group (whose b and c it keeps in LDS), so groups
// of fewer channels, or of some more than a multiple, leave lanes without work: groups of 4 seven of eight.
template <int L>
struct Place {
    int channel, group, own;
    bool live;
    __device__ __forceinline__ Place(const ScanCall& c, int tile) {
        const int per = c.channels / c.groups, tiles = (per + kScanSlice - 1) / kScanSlice;
        group = tile / tiles;
        const int at = tile % tiles * kScanSlice + threadIdx.x / L;
        live = at < per;
        channel = group * per + (live ? at : per - 1);
        own = threadIdx.x % L;
    }
};

template <class T>
__device__ __forceinline__ const T* row(const TokenRows& r, int t) { return (const T*)r.p + (int64_t)t * r.ts; }
template <class T>
__device__ __forceinline__ T* row_out(const TokenRows& r, int t) { return (T*)r.p + (int64_t)t * r.ts; }

// A lane's tokens of a tile, `mine` + i: from the tile's row i, which is the same for the workgroup, by an offset that stays (rows are less than 16 MiB
// apart, and 60 of them less than 1 GiB).
template <class T>
struct Column {
    const TokenRows rows;
    const unsigned here, off;
    __device__ __forceinline__ Column(const TokenRows& r, int channel, int mine)
        : rows(r), here(channel * (unsigned)sizeof(T)), off(here + (unsigned)(mine * (int)r.ts) * (unsigned)sizeof(T)) {}
    // (what lies behind the last token is read from the tile's own row instead)
    __device__ __forceinline__ T load(int t0, int i, int last, bool in) const {
        return *(const T*)((const char*)row<T>(rows, min(t0 + i, last)) + (in ? off : here));
    }
    __device__ __forceinline__ void store(int t0, int i, float v) const { *(T*)((char*)row_out<T>(rows, t0 + i) + off) = Traits<T>::from_f32(v); }
};

template <int S>
__device__ __forceinline__ void load_states(float (&to)[S], const float* p) { __builtin_memcpy(to, __builtin_assume_aligned(p, 4), S * 4); }
template <int S>
__device__ __forceinline__ void store_states(float* p, const float (&from)[S]) { __builtin_memcpy(__builtin_assume_aligned(p, 4), from, S * 4); }
enum Pass { kWhole, kSums, kMarks, kSumsBoth };

// b and c of some tokens in fp32 in LDS, a state's tokens next to each other, so that a lane reads four tokens of a state at once.  The rows of the states that
// the lanes of a channel read at once follow each other, four words beyond a multiple of the banks.
template <class T, int N, int L, bool WITH_C>
struct Shared {
    static constexpr int kThreads = kScanSlice * L, kTokens = 4 * L, kRow = kTokens + 4, kQuads = N / 4, kMaps = WITH_C ? 2 : 1;
    static constexpr int kPieces = kTokens * kQuads * kMaps, kEach = (kPieces + kThreads - 1) / kThreads;
    typedef float Room[kMaps][N][kRow];
    static __device__ __forceinline__ int row_of(int lane, int s) { return s * L + lane; }     // of state lane * (N / L) + s
    Piece<T, 4> piece[kEach];
    // tokens from t0 to last of a group's rows (zeros behind them)
    __device__ __forceinline__ void fetch(const ScanCall& call, int group, int t0, int last) {
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            const int e = threadIdx.x + k * kThreads, map = e / (kTokens * kQuads), t = t0 + e / kQuads % kTokens;
            piece[k].clear();
            if (e < kPieces && t <= last) piece[k].load(row<T>(map ? call.c : call.b, t) + group * N + e % kQuads * 4);
        }
    }
    __device__ __forceinline__ void park(Room& room) const {
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            const int e = threadIdx.x + k * kThreads, map = e / (kTokens * kQuads), t = e / kQuads % kTokens;
            if (e >= kPieces) continue;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int n = e % kQuads * 4 + i;
                room[map][row_of(n / (N / L), n % (N / L))][t] = piece[k].at(i);
            }
        }
    }
};

// kWhole: outputs and the last state.  kSums: a slot's state from zero and the sum of its steps.  For the gradient, the state in front of every L tokens
// (a mark): kMarks, of sequences that are not cut; kSumsBoth, from zero, with the sum of the steps so far, what kSums has, and what the slot adds to the gradient of
// the state in front of it.
//
// L lanes have a channel, with S states each: kScanSlice channels a workgroup, so that a compute unit has two of them, which do not wait at the
// same time (where a lane has no more than 128 registers: fp32 with 64 states takes 130, kSumsBoth with 64 states 134 to 142, and of those a unit has one).
// Tokens go by in tiles of 4 L.  A tile is loaded with a lane to a channel and four tokens, so that rows are read whole (with the lanes as they share channels, every
// lane was an access of its own, and those bounded the kernel), what the states need of them goes through LDS, and so do the outputs back, in the steps' places.
template <class T, int L, int S, int PASS>
__global__ void __launch_bounds__(kScanSlice * L) scan_kernel(ScanCall call, int tiles) {
    constexpr int N = L * S;
    constexpr bool kWithC = PASS == kWhole || PASS == kSumsBoth, kFromZero = PASS == kSums || PASS == kSumsBoth, kMark = PASS == kMarks || PASS == kSumsBoth;
    typedef Shared<T, N, L, kWithC> Tile;
    constexpr int kTokens = Tile::kTokens, kRow = Tile::kRow;
    __shared__ __align__(16) typename Tile::Room room;
    __shared__ __align__(16) float own[PASS == kSumsBoth ? 3 : 2][kScanSlice][kRow];         // steps (outputs), steps times x, dy
    const int64_t slot_number = blockIdx.x / tiles;
    const Slot slot = slot_at(call.slots, (int)slot_number);
    if (!slot.used) return;
    if (PASS == kSums && slot.last) return;         // (what a sequence's last slot leaves of a state nobody asks for)
    const Place<L> me(call, blockIdx.x % tiles);
    const int64_t state_at = (int64_t)me.channel * N + me.own * S, per_state = (int64_t)call.channels * N;
    float a[S], h[S];
    load_states(a, call.a + state_at);
#pragma unroll
    for (int s = 0; s < S; ++s) a[s] = rate_of(a[s]);
#pragma unroll
    for (int s = 0; s < S; ++s) h[s] = 0.0f;
    if constexpr (!kFromZero) {
        // (only a whole sequence reads its initial state here: of one that is cut, the last slot may write the final state over it meanwhile)
        if (!slot.first || !slot.last) load_states(h, call.states_at + slot_number * per_state + state_at);
        else if (call.initial) load_states(h, call.initial + slot.sequence * per_state + state_at);
    }
    int64_t mark = 0;
    if constexpr (kMark) mark = first_slot(call.marks, slot.sequence) + (slot.from - slot.lo) / L;
    float passed = 0.0f;                // the steps so far (kSumsBoth)
    float along[S], reach[S];           // exp(a * the steps so far), and the sum of that times c dy
#pragma unroll
    for (int s = 0; s < S; ++s) along[s] = 1.0f, reach[s] = 0.0f;
    const int last = slot.until - 1;

    // a lane's channel as tiles are loaded, and its four tokens of a tile
    const int per = call.channels / call.groups, first = blockIdx.x % tiles % ((per + kScanSlice - 1) / kScanSlice) * kScanSlice;
    const int lane = threadIdx.x % kScanSlice, run = threadIdx.x / kScanSlice, mine = 4 * run;
    const bool live = first + lane < per;
    const int channel = me.group * per + (live ? first + lane : per - 1);
    const bool gated = call.gate.p != nullptr, soft = call.softplus != 0;
    const float bias = call.bias ? call.bias[channel] : 0.0f, skip = call.skip ? call.skip[channel] : 0.0f;
    const Column<T> xs(call.x, channel, mine), deltas(call.delta, channel, mine), gates(call.gate, channel, mine), d_outs(call.d_out, channel, mine),
        outs(call.out, channel, mine);
    struct Tokens { T x[4], delta[4], gate[4], d_out[4]; } next;
    auto fetch = [&](int t0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool in = t0 + mine + i <= last;
            next.x[i] = xs.load(t0, i, last, in);
            next.delta[i] = deltas.load(t0, i, last, in);
            if constexpr (kWithC)
                if (gated) next.gate[i] = gates.load(t0, i, last, in);
            if constexpr (PASS == kSumsBoth) next.d_out[i] = d_outs.load(t0, i, last, in);
        }
    };
    Tile tile;
    float steps = 0.0f;
    if (slot.from <= last) {
        tile.fetch(call, me.group, slot.from, last);
        fetch(slot.from);
    }
    for (int t0 = slot.from; t0 <= last; t0 += kTokens) {
        f32x4 step, add, dy, past, through;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool in = t0 + mine + i <= last;          // (tokens behind the last one: a step of nothing, and b and c of zero)
            const float x = Traits<T>::to_f32(next.x[i]), pre = Traits<T>::to_f32(next.delta[i]) + bias, full = soft ? softplus_of(pre) : pre;
            step[i] = in ? full : 0.0f;
            add[i] = in ? full * x : 0.0f;
            past[i] = skip * x;
            through[i] = 1.0f;
            if constexpr (kWithC) {
                if (gated) {
                    const float z = Traits<T>::to_f32(next.gate[i]);
                    through[i] = z * sigmoid_of(z);
                }
            }
            if constexpr (PASS == kSumsBoth) dy[i] = in ? Traits<T>::to_f32(next.d_out[i]) * through[i] : 0.0f;
            steps += step[i];
        }
        *(f32x4*)&own[0][lane][mine] = step;
        *(f32x4*)&own[1][lane][mine] = add;
        if constexpr (PASS == kSumsBoth) *(f32x4*)&own[2][lane][mine] = dy;
        tile.park(room);
        __syncthreads();
        if (t0 + kTokens <= last) {
            tile.fetch(call, me.group, t0 + kTokens, last);
            fetch(t0 + kTokens);
        }
        const int channel_at = threadIdx.x / L;
#pragma unroll PASS == kWhole ? 4 : 1
        for (int block = 0; block < kTokens; block += L) {
            if constexpr (kMark) {
                if (t0 + block <= last && me.live) {
                    store_states(call.marks_at + mark * per_state + state_at, h);
                    if (PASS == kSumsBoth && me.own == 0) call.mark_steps_at[mark * call.channels + me.channel] = passed;
                }
                ++mark;
            }
            float sums[L];
#pragma unroll
            for (int f = 0; f < L; f += 4) {
                const f32x4 ti = *(const f32x4*)&own[0][channel_at][block + f], ui = *(const f32x4*)&own[1][channel_at][block + f];
                f32x4 dyi, b[S], c[S];
                if constexpr (PASS == kSumsBoth) {
                    dyi = *(const f32x4*)&own[2][channel_at][block + f];
                    passed += (ti[0] + ti[1]) + (ti[2] + ti[3]);
                }
#pragma unroll
                for (int s = 0; s < S; ++s) {
                    b[s] = *(const f32x4*)&room[0][Tile::row_of(me.own, s)][block + f];
                    if constexpr (kWithC) c[s] = *(const f32x4*)&room[1][Tile::row_of(me.own, s)][block + f];
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float y = 0.0f;
#pragma unroll
                    for (int s = 0; s < S; ++s) {
                        const float keep = exp2_of(ti[i] * a[s]);
                        h[s] = fmaf(keep, h[s], ui[i] * b[s][i]);
                        if constexpr (PASS == kWhole) y = s == 0 ? c[s][i] * h[s] : fmaf(c[s][i], h[s], y);
                        if constexpr (PASS == kSumsBoth) {
                            along[s] *= keep;
                            reach[s] = fmaf(along[s] * dyi[i], c[s][i], reach[s]);
                        }
                    }
                    sums[f + i] = y;
                }
                // (b and c of the next four tokens stay in LDS until these are done: their registers are wanted)
                if constexpr (S > 1) __builtin_amdgcn_sched_barrier(0);
            }
            if constexpr (PASS == kWhole) own[0][channel_at][block + me.own] = deal<L>(sums, me.own);
        }
        __syncthreads();
        if constexpr (PASS == kWhole) {
            const f32x4 y = *(const f32x4*)&own[0][lane][mine];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (t0 + mine + i <= last && live) outs.store(t0, i, (y[i] + past[i]) * through[i]);
        }
    }
    if constexpr (PASS == kWhole) {
        if (call.final_state && slot.last && me.live) store_states(call.final_state + slot.sequence * per_state + state_at, h);
    } else if constexpr (kFromZero) {
        const int64_t at = slot_number * per_state + state_at;
        if (me.live) {
            store_states(call.states_at + at, h);
            if constexpr (PASS == kSumsBoth) store_states(call.d_states_at + at, reach);
        }
        // (each has the steps of its own tokens)
        own[0][lane][run] = steps;
        __syncthreads();
        if (run == 0 && live) {
#pragma unroll
            for (int r = 1; r < L; ++r) steps += own[0][lane][r];
            call.steps_at[slot_number * call.channels + channel] = steps;
        }
    }
}

// The state that each slot of a sequence that is cut starts from, and (BOTH) the state's gradient behind each, in the places of the slots' own sums.  A thread has one state of a sequence; the next slots' sums are on their way while one is joined.
template <bool BOTH>
__global__ void __launch_bounds__(256) scan_join_kernel(ScanCall call, int blocks) {
    const int b = blockIdx.x / blocks;
    const int64_t per_state = (int64_t)call.channels * call.states, at = (int64_t)(blockIdx.x % blocks) * 256 + threadIdx.x;
    if (at >= per_state) return;
    int lo, hi;
    rows_of_sequence(call.slots, b, lo, hi);
    const int64_t from = first_slot(call.slots, b), count = ((int64_t)hi - lo + call.slots.run - 1) / call.slots.run;
    if (count < 2) return;
    const float a = rate_of(call.a[at]);
    const int64_t channel = at / call.states;
    constexpr int kAhead = 8;
    // over slots in the order that `slot_of` gives; v goes to the first, and on
    auto join = [&](float* sums, float v, auto slot_of) {
        for (int64_t k0 = 0; k0 < count - 1; k0 += kAhead) {
            float own[kAhead], steps[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int64_t slot = from + slot_of(min(k0 + k, count - 2));
                own[k] = sums[slot * per_state + at];
                steps[k] = call.steps_at[slot * call.channels + channel];
            }
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
                if (k0 + k < count - 1) {
                    sums[(from + slot_of(k0 + k)) * per_state + at] = v;
                    v = fmaf(exp2_of(a * steps[k]), v, own[k]);
                }
        }
        sums[(from + slot_of(count - 1)) * per_state + at] = v;
    };
    join(call.states_at, call.initial ? call.initial[b * per_state + at] : 0.0f, [](int64_t k) { return k; });
    if constexpr (BOTH) join(call.d_states_at, call.d_final ? call.d_final[b * per_state + at] : 0.0f, [&](int64_t k) { return count - 1 - k; });
}

// A slot of the gradient, with the scan's lanes and tiles, the last tile first.  Of every L tokens the states come from their mark, stay in registers, and
// the state's gradient goes back over them.
template <class T, int L, int S>
__global__ void __launch_bounds__(kScanSlice * L) scan_backward_kernel(ScanCall call, int tiles) {
    constexpr int N = L * S, kThreads = kScanSlice * L, kWaves = kThreads / 64, kSums = L * 2 * N;
    typedef Shared<T, N, L, true> Tile;
    constexpr int kTokens = Tile::kTokens, kRow = Tile::kRow;
    // a window's sums over the channels of a wave: one place, or two that take turns, which save a barrier
    constexpr int kTurns = S == 1 ? 2 : 1;
    constexpr bool kTileAhead = S < 4;          // (four states a lane leave no registers for it)
    __shared__ __align__(16) typename Tile::Room room;
    __shared__ __align__(16) float own[3][kScanSlice][kRow];        // steps (y), steps times x (e), dy (the sum of w a)
    __shared__ float sums[kTurns][kWaves][kSums];
    const int64_t slot_number = blockIdx.x / tiles;
    const Slot slot = slot_at(call.slots, (int)slot_number);
    const Place<L> me(call, blockIdx.x % tiles);
    const int64_t state_at = (int64_t)me.channel * N + me.own * S, per_state = (int64_t)call.channels * N;
    float* parts = call.parts_at + slot_number * (per_state + 2 * call.channels);
    float d_a[S], of_tile[S], carry[S], a[S], start[S];      // (of_tile: d_a of a tile's tokens, so that long sequences add up tiles and not tokens)
#pragma unroll
    for (int s = 0; s < S; ++s) d_a[s] = of_tile[s] = carry[s] = start[s] = 0.0f;
    load_states(a, call.a + state_at);
#pragma unroll
    for (int s = 0; s < S; ++s) a[s] = rate_of(a[s]);
    // (lanes without a channel read another's values, and must not add even an infinity to sums)
    if (me.live && slot.used) {
        const bool whole = slot.first && slot.last;
        if (!whole) load_states(carry, call.d_states_at + slot_number * per_state + state_at);
        else if (call.d_final) load_states(carry, call.d_final + slot.sequence * per_state + state_at);
        if (call.cut) {             // (marks are of a slot from zero: what it started from comes on top)
            if (!whole) load_states(start, call.states_at + slot_number * per_state + state_at);
            else if (call.initial) load_states(start, call.initial + slot.sequence * per_state + state_at);
        }
    }
    const int last = slot.until - 1;

    // a lane's channel as tiles are loaded, and its four tokens of a tile
    const int per = call.channels / call.groups, first = blockIdx.x % tiles % ((per + kScanSlice - 1) / kScanSlice) * kScanSlice;
    const int lane = threadIdx.x % kScanSlice, run = threadIdx.x / kScanSlice, mine = 4 * run;
    const bool live = first + lane < per;
    const int channel = me.group * per + (live ? first + lane : per - 1);
    const bool gated = call.gate.p != nullptr, soft = call.softplus != 0;
    const float bias = call.bias ? call.bias[channel] : 0.0f, skip = call.skip ? call.skip[channel] : 0.0f;
    float d_skip = 0.0f, d_bias = 0.0f;
    const Column<T> xs(call.x, channel, mine), deltas(call.delta, channel, mine), gates(call.gate, channel, mine), d_outs(call.d_out, channel, mine),
        d_xs(call.d_x, channel, mine), d_deltas(call.d_delta, channel, mine), d_gates(call.d_gate, channel, mine);
    struct Tokens { T x[4], delta[4], gate[4], d_out[4]; } next;
    Tile tile;
    auto fetch = [&](int t0) {
        tile.fetch(call, me.group, t0, last);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool in = t0 + mine + i <= last;
            next.x[i] = xs.load(t0, i, last, in);
            next.delta[i] = deltas.load(t0, i, last, in);
            if (gated) next.gate[i] = gates.load(t0, i, last, in);
            next.d_out[i] = d_outs.load(t0, i, last, in);
        }
    };
    const int64_t marks = first_slot(call.marks, slot.sequence);
    const int channel_at = threadIdx.x / L, wave_lane = threadIdx.x & 63;
    const int behind = slot.used ? (slot.until - slot.from + kTokens - 1) / kTokens : 0;
    // the mark of the window in front of the one that is worked on
    float ahead[S], passed = 0.0f;
    auto ask = [&](int t) {
        const int64_t at = marks + (max(t, slot.from) - slot.lo) / L;
        load_states(ahead, call.marks_at + at * per_state + state_at);
        if (call.cut) passed = call.mark_steps_at[at * call.channels + me.channel];
    };
    if (behind > 0) {
        if constexpr (kTileAhead) fetch(slot.from + (behind - 1) * kTokens);
        ask(slot.from + (last - slot.from) / L * L);
    }
    int turn = 0;
    for (int n = behind - 1; n >= 0; --n) {
        const int t0 = slot.from + n * kTokens;
        if constexpr (!kTileAhead) fetch(t0);
        const Tokens now = next;
        f32x4 step, add, dy;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool in = t0 + mine + i <= last && live;         // (others: a step of nothing, and no gradient)
            const float x = Traits<T>::to_f32(now.x[i]), pre = Traits<T>::to_f32(now.delta[i]) + bias, full = soft ? softplus_of(pre) : pre;
            float back = Traits<T>::to_f32(now.d_out[i]);
            if (gated) {
                const float z = Traits<T>::to_f32(now.gate[i]);
                back *= z * sigmoid_of(z);
            }
            step[i] = in ? full : 0.0f;
            add[i] = in ? full * x : 0.0f;
            dy[i] = in ? back : 0.0f;
        }
        *(f32x4*)&own[0][lane][mine] = step;
        *(f32x4*)&own[1][lane][mine] = add;
        *(f32x4*)&own[2][lane][mine] = dy;
        tile.park(room);
        __syncthreads();
        if (kTileAhead && n > 0) fetch(t0 - kTokens);
#pragma unroll 1
        for (int base = kTokens - L; base >= 0; base -= L) {
            const int from = t0 + base;
            if (from > last) continue;
            float mark[S];
#pragma unroll
            for (int s = 0; s < S; ++s) {
                mark[s] = call.cut ? fmaf(exp2_of(passed * a[s]), start[s], ahead[s]) : ahead[s];
                if (!me.live) mark[s] = 0.0f;
            }
            ask(from - L);
            float states[L][S], keeps[S == 1 ? L : 1][S], sum[L], sum2[L];
            float h[S];
#pragma unroll
            for (int s = 0; s < S; ++s) h[s] = mark[s];
#pragma unroll
            for (int f = 0; f < L; f += 4) {
                const f32x4 ti = *(const f32x4*)&own[0][channel_at][base + f], ui = *(const f32x4*)&own[1][channel_at][base + f];
                f32x4 b[S], c[S];
#pragma unroll
                for (int s = 0; s < S; ++s) {
                    b[s] = *(const f32x4*)&room[0][Tile::row_of(me.own, s)][base + f];
                    c[s] = *(const f32x4*)&room[1][Tile::row_of(me.own, s)][base + f];
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float y = 0.0f;
#pragma unroll
                    for (int s = 0; s < S; ++s) {
                        const float keep = exp2_of(ti[i] * a[s]);
                        if constexpr (S == 1) keeps[f + i][s] = keep;
                        states[f + i][s] = h[s] = fmaf(keep, h[s], ui[i] * b[s][i]);
                        y = s == 0 ? c[s][i] * h[s] : fmaf(c[s][i], h[s], y);
                    }
                    sum[f + i] = y;
                }
                if constexpr (S > 1) __builtin_amdgcn_sched_barrier(0);
            }
            const float y = gated ? deal<L>(sum, me.own) : 0.0f;
            float(&place)[kSums] = sums[turn][threadIdx.x >> 6];
#pragma unroll
            for (int f = L - 4; f >= 0; f -= 4) {
                const f32x4 ti = *(const f32x4*)&own[0][channel_at][base + f], ui = *(const f32x4*)&own[1][channel_at][base + f];
                const f32x4 dyi = *(const f32x4*)&own[2][channel_at][base + f];
                f32x4 b[S], c[S];
                float both[4][S];
#pragma unroll
                for (int s = 0; s < S; ++s) {
                    b[s] = *(const f32x4*)&room[0][Tile::row_of(me.own, s)][base + f];
                    c[s] = *(const f32x4*)&room[1][Tile::row_of(me.own, s)][base + f];
                }
#pragma unroll
                for (int i = 3; i >= 0; --i) {
                    const int t = f + i;
                    float e = 0.0f, along = 0.0f;
#pragma unroll
                    for (int s = 0; s < S; ++s) {
                        const float dh = fmaf(c[s][i], dyi[i], carry[s]);
                        both[i][s] = halve32(dh * ui[i], dyi[i] * states[t][s]);
                        e = s == 0 ? dh * b[s][i] : fmaf(dh, b[s][i], e);
                        const float keep = S == 1 ? keeps[S == 1 ? t : 0][s] : exp2_of(ti[i] * a[s]);
                        carry[s] = keep * dh;
                        const float through = carry[s] * (t > 0 ? states[t > 0 ? t - 1 : 0][s] : mark[s]);
                        of_tile[s] = fmaf(through, ti[i], of_tile[s]);
                        along = s == 0 ? through * a[s] : fmaf(through, a[s], along);
                    }
                    sum[t] = e;
                    sum2[t] = along;
                }
                // sums over the channels of the wave: a lane ends up with those of b or of c (its 32), of one token of two (its 16), or of four (its 8)
                const int of = (wave_lane & 32 ? N : 0) + me.own * S;
#pragma unroll
                for (int s = 0; s < S; ++s) {
                    const float lower = halve16(both[0][s], both[1][s]), higher = halve16(both[2][s], both[3][s]);
                    const int odd = wave_lane & 16 ? 1 : 0;
                    if constexpr (L == 16) {
                        place[(f + odd) * 2 * N + of + s] = lower;
                        place[(f + 2 + odd) * 2 * N + of + s] = higher;
                    } else {
                        place[(f + odd + (wave_lane & 8 ? 2 : 0)) * 2 * N + of + s] = halve8(lower, higher, wave_lane);
                    }
                }
                if constexpr (S > 1) __builtin_amdgcn_sched_barrier(0);
            }
            const float e = deal<L>(sum, me.own), along = deal<L>(sum2, me.own);
            own[0][channel_at][base + me.own] = y;
            own[1][channel_at][base + me.own] = e;
            own[2][channel_at][base + me.own] = along;
            __syncthreads();
            const int count = min(L, last - from + 1) * 2 * N;
            float* to = call.shared_at + ((int64_t)(blockIdx.x % tiles) * call.slots.tokens + from) * (2 * N);
            for (int k = threadIdx.x; k < count; k += kThreads) {
                float v = sums[turn][0][k];
#pragma unroll
                for (int o = 1; o < kWaves; ++o) v += sums[turn][o][k];
                to[k] = v;
            }
            if constexpr (kTurns == 2) turn ^= 1;
            else __syncthreads();
        }
#pragma unroll
        for (int s = 0; s < S; ++s) {
            d_a[s] += of_tile[s];
            of_tile[s] = 0.0f;
        }
        const f32x4 y = *(const f32x4*)&own[0][lane][mine], e = *(const f32x4*)&own[1][lane][mine], along = *(const f32x4*)&own[2][lane][mine];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (t0 + mine + i > last || !live) continue;
            const float x = Traits<T>::to_f32(now.x[i]);
            float d_step = fmaf(x, e[i], kLn2 * along[i]);
            if (soft) d_step *= sigmoid_of(Traits<T>::to_f32(now.delta[i]) + bias);
            d_xs.store(t0, i, fmaf(step[i], e[i], skip * dy[i]));
            d_deltas.store(t0, i, d_step);
            if (gated) {
                const float z = Traits<T>::to_f32(now.gate[i]), open = sigmoid_of(z);
                d_gates.store(t0, i, Traits<T>::to_f32(now.d_out[i]) * fmaf(skip, x, y[i]) * (open * fmaf(z, 1.0f - open, 1.0f)));
            }
            d_skip = fmaf(dy[i], x, d_skip);
            d_bias += d_step;
        }
    }
    if (slot.used && slot.first && call.d_initial && me.live) store_states(call.d_initial + slot.sequence * per_state + state_at, carry);
    if (me.live) store_states(parts + state_at, d_a);
    // (each has the sums of its own tokens; the places that they go to hold the last tile's y and e, which other waves may be reading still)
    __syncthreads();
    own[0][lane][run] = d_skip;
    own[1][lane][run] = d_bias;
    __syncthreads();
    if (run == 0 && live) {
#pragma unroll
        for (int r = 1; r < L; ++r) {
            d_skip += own[0][lane][r];
            d_bias += own[1][lane][r];
        }
        parts[per_state + channel] = d_skip;
        parts[per_state + call.channels + channel] = d_bias;
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
    y = sum_of_four(y);
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

// The lanes that share a channel, and the states of each, of the passes over whole sequences.
template <class F>
hipError_t with_lanes(int states, F&& f) {
    using std::integral_constant;
    switch (states) {
        case 8: return f(integral_constant<int, 8>{}, integral_constant<int, 1>{});
        case 16: return f(integral_constant<int, 16>{}, integral_constant<int, 1>{});
        case 32: return f(integral_constant<int, 16>{}, integral_constant<int, 2>{});
        case 64: return f(integral_constant<int, 16>{}, integral_constant<int, 4>{});
    }
    return hipErrorInvalidValue;
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
        return with_lanes(c.states, [&](auto l, auto s) {
            constexpr int L = decltype(l)::value, S = decltype(s)::value;
            const int tiles = scan_tiles(c.channels, c.groups);
            const dim3 grid((unsigned)(slot_count(c.slots) * tiles)), threads(kScanSlice * L);
            if (c.cut) {
                hipLaunchKernelGGL((scan_kernel<T, L, S, kSums>), grid, threads, 0, stream, c, tiles);
                hipError_t e = hipGetLastError();
                if (e == hipSuccess) e = join<false>(c, stream);
                if (e != hipSuccess) return e;
            }
            hipLaunchKernelGGL((scan_kernel<T, L, S, kWhole>), grid, threads, 0, stream, c, tiles);
            return hipGetLastError();
        });
    });
}

hipError_t launch_scan_backward(int dt, const ScanCall& c, hipStream_t stream) {
    return with_type(dt, [&](auto type) {
        typedef decltype(type) T;
        return with_lanes(c.states, [&](auto l, auto s) {
            constexpr int L = decltype(l)::value, S = decltype(s)::value;
            const int tiles = scan_tiles(c.channels, c.groups);
            const int64_t slots = slot_count(c.slots);
            const dim3 grid((unsigned)(slots * tiles)), threads(kScanSlice * L);
            if (c.cut) hipLaunchKernelGGL((scan_kernel<T, L, S, kSumsBoth>), grid, threads, 0, stream, c, tiles);
            else hipLaunchKernelGGL((scan_kernel<T, L, S, kMarks>), grid, threads, 0, stream, c, tiles);
            hipError_t e = hipGetLastError();
            if (e == hipSuccess && c.cut) e = join<true>(c, stream);
            if (e != hipSuccess) return e;
            hipLaunchKernelGGL((scan_backward_kernel<T, L, S>), grid, threads, 0, stream, c, tiles);
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
