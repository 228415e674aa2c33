// The gated linear recurrence: S_i = a_i S_{i-1} + k_i v_i^T, o_i = scale q_i^T S_i, a_i = exp(log_gate_i).
//
// In chunks of 64 tokens, with F the running sum of the gates' logarithms inside a chunk and S the state before it,
//     o_i = scale ( sum_{j <= i} e^{F_i - F_j} (q_i . k_j) v_j  +  e^{F_i} q_i^T S ),       S <- e^{F_end} S + sum_j e^{F_end - F_j} k_j v_j^T,
// all of it 16x16 matrix instructions; no exponent is above 0 where no gate is (but for the factor that the state is kept with, see Gates).
//
// The gradient is the same scan three times.  With dS the gradient that arrives at a state:
//     dq_i = scale ( sum_{j <= i} e^{..} (do_i . v_j) k_j + e^{F_i} do_i^T S^T )        the scan with (do; v, k) for (q; k, v)
//     dk_j = scale   sum_{i >= j} e^{..} (v_j . do_i) q_i + e^{..} v_j^T dS^T           the scan from the end with (v; do, q)
//     dv_j = scale   sum_{i >= j} e^{..} (k_j . q_i) do_i + e^{..} k_j^T dS             the scan from the end with (k; q, do)
// From the end means: rows of a chunk in the opposite order, running sums that leave a row's own gate out.  And
//     d log_gate_t = sum_{i >= t} (q_i . dq_i - k_i . dk_i) + <dS_end, S_end>           over the tokens up to any later border "end",
// because what flows over the border before t is what leaves the tokens before it and reaches t or later ones.
//
// Long sequences are cut into segments, so that the GPU is full: a first pass sums each segment's own contribution to the state, a
// second joins them in order (a few numbers a state), and the scan starts every segment from its state.  Where a segment holds a whole
// sequence the first two are not launched.
#include "recurrence_tile.h"
#include "msla_sequence_kernels.h"

namespace msla {
namespace rec {

constexpr int kThreads = 256;        // of the kernels that have no tiles

struct SweepArgs {
    Heads a, b, c;                  // (q; k, v) and its permutations
    char* out;
    long out_ts, out_hs;            // bytes
    Heads m;                        // like out: masks it where m.relu is set, and dots[token, head, slice] = m . out
    float* dots;
    const void* gate;
    long gate_ts;
    const float* start;             // states that segments start from [slot, heads_kv, d, d] (NULL: `first`)
    const float* first;             // ... that sequences start from [sequence, heads_kv, d, d] (NULL: zero)
    float* last;                    // ... that sequences end with (NULL: not wanted)
    int rs;                         // 1: a state's rows (channels of a) lie next to each other in memory; d: its columns (channels of out)
    Layout layout;
    int heads, ga, gb, reverse;     // state heads; heads of a and of (b, c) to each
    float score_scale, in_scale, weight_scale;
};

struct StateArgs {
    Heads b, c;
    const void* gate;
    long gate_ts;
    float* own;                     // [slot, heads_kv, d, d]
    float* decay;                   // [slot, heads_kv]
    int rs;                         // as above, of rows of channels of b and columns of channels of c
    Layout layout;
    int heads, gb, reverse;
    float weight_scale;
};

// Bounds on the magnitudes of a tile's rows of one head, from what the waves left in LDS (fp16 alone): [wave][head][a, b, c].  A head's own, so that
// its precision does not hang on the heads that share its workgroup.
template <class Ti>
__device__ __forceinline__ float tile_top(const unsigned* top, int head) {
    unsigned t = top[3 * head];
#pragma unroll
    for (int w = 1; w < Ti::kWaves; ++w) t = max(t, top[3 * (w * Ti::kHeads + head)]);
    return half_bits(t);
}

// `mine`: of this lane's pieces, which are all of one head (Tile::head_of)
template <class Ti>
__device__ __forceinline__ void leave_top(unsigned* top, unsigned mine) {
    const int lane = lane_id();
    top += 3 * Ti::kHeads * (threadIdx.x >> 6);
    if constexpr (Ti::kHeads == 1) {
        mine = running_max(mine);
        if (lane == 63) *top = mine;
    } else {
        // lanes 8 apart have the same head, and so have two (heads of 16) or four (of 32) neighbours
        constexpr int kLanes = Ti::kPerRow / Ti::kHeads;
        static_assert(Ti::kPerRow == 8 && (kLanes == 2 || kLanes == 4), "eight pieces a row");
        mine = max(mine, moved<0x128, 0xf>(mine));              // row_ror 8
        const u32x2 rows = __builtin_amdgcn_permlane16_swap(mine, mine, false, false);
        mine = max(rows[0], rows[1]);
        const u32x2 halves = __builtin_amdgcn_permlane32_swap(mine, mine, false, false);
        mine = max(halves[0], halves[1]);
        mine = max(mine, moved<0xb1, 0xf>(mine));               // quad_perm 1 0 3 2
        if constexpr (kLanes == 4) mine = max(mine, moved<0x4e, 0xf>(mine));    // quad_perm 2 3 0 1
        if (lane < 8 && lane % kLanes == 0) top[3 * (lane / kLanes)] = mine;
    }
}

// The state's part of a wave: rows are all channels of the key, columns the wave's 16 output channels.
template <class T, int D>
struct State {
    typedef Tile<T, D> Ti;
    f32x4 s[Ti::kBlocks];

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int b = 0; b < Ti::kBlocks; ++b) s[b] = f32x4{0, 0, 0, 0};
    }
    // In memory a row's or (rs == 1) a column's elements lie next to each other: a lane's four rows are then one access.
    template <class F>
    __device__ __forceinline__ void blocks(int slice, F&& f) {
        const int x = lane_id() & 15, q = lane_id() >> 4;
#pragma unroll
        for (int b = 0; b < Ti::kBlocks; ++b) f(s[b], Ti::channel(b, 4 * q), slice + x);
    }
    __device__ __forceinline__ void read(const float* p, int slice, int rs) {
        if (rs == 1)
            blocks(slice, [&](f32x4& v, int row, int col) { v = *(const f32x4*)(p + (unsigned)(row + col * D)); });
        else
            blocks(slice, [&](f32x4& v, int row, int col) {
#pragma unroll
                for (int r = 0; r < 4; ++r) v[r] = p[(unsigned)((row + r) * D + col)];
            });
    }
    __device__ __forceinline__ void write(float* p, int slice, int rs, float unit) {
        scale(unit);
        if (rs == 1)
            blocks(slice, [&](f32x4& v, int row, int col) { *(f32x4*)(p + (unsigned)(row + col * D)) = v; });
        else
            blocks(slice, [&](f32x4& v, int row, int col) {
#pragma unroll
                for (int r = 0; r < 4; ++r) p[(unsigned)((row + r) * D + col)] = v[r];
            });
    }
    __device__ __forceinline__ void scale(float f) {
#pragma unroll
        for (int b = 0; b < Ti::kBlocks; ++b)
#pragma unroll
            for (int r = 0; r < 4; ++r) s[b][r] *= f;
    }
    __device__ __forceinline__ float top() const {
        float t = 0.0f;
#pragma unroll
        for (int b = 0; b < Ti::kBlocks; ++b)
#pragma unroll
            for (int r = 0; r < 4; ++r) t = fmaxf(t, fabsf(s[b][r]));
#pragma unroll
        for (int d = 1; d < 64; d *= 2) t = fmaxf(t, __shfl_xor(t, d));
        return t;
    }
    // step b's channels as an operand, in parts
    __device__ __forceinline__ void operand(int b, float f, typename Ti::Op (&part)[kParts<T>]) const {
        float v[Ti::kOp];
#pragma unroll
        for (int e = 0; e < Ti::kOp; ++e) v[e] = s[b * Ti::kJoinOp + e / 4][e % 4] * f;
        Ti::template split<kParts<T>>(v, part);
    }
    // += sum_j b_j (w_j c_j)^T over the chunk; vt: the wave's columns of c over tokens.
    __device__ __forceinline__ void add(char* tb, const typename Ti::Vec (&vt)[Ti::kTokenSteps], const float* weight, float unit) {
        const int lane = lane_id_again(), x = lane & 15, q = lane >> 4;
#pragma unroll
        for (int st = 0; st < Ti::kTokenSteps; ++st) {
            __builtin_amdgcn_sched_barrier(0);
            // (operands are on their way while others' products run)
            typename Ti::Vec kt = Ti::key_operand(tb, 0, st, x, q);
            float v[Ti::kVec];
#pragma unroll
            for (int j = 0; j < Ti::kJoin; ++j) {
                const f32x4 f = *(const f32x4*)(weight + st * Ti::kTokenStep + 16 * j + 4 * q);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    v[4 * j + r] = Ti::Tr::to_f32(vt[st][4 * j + r]) * f[r];
                    if constexpr (Ti::kNormalise) v[4 * j + r] *= unit;
                }
            }
            typename Ti::Vec part[kParts<T>];
            Ti::template split<kParts<T>>(v, part);
#pragma unroll
            for (int b = 0; b < Ti::kBlocks; b += 2) {
                typename Ti::Vec more = kt, next = kt;
                if (b + 1 < Ti::kBlocks) more = Ti::key_operand(tb, b + 1, st, x, q);
                if (b + 2 < Ti::kBlocks) next = Ti::key_operand(tb, b + 2, st, x, q);
#pragma unroll
                for (int p = 0; p < kParts<T>; ++p) {
                    s[b] = Ti::Tr::mma_vec(s[b], kt, part[p]);
                    if (b + 1 < Ti::kBlocks) s[b + 1] = Ti::Tr::mma_vec(s[b + 1], more, part[p]);
                }
                kt = next;
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
};

// A chunk's gates, a lane's row each, as they stand in memory: what is done with them waits for them, so that is left for when they are
// needed.  Like the tiles: from a lowest address, 0 where there is no row.
template <class T>
struct GateRows {
    const T* at;
    long ts;
    int live;
    __device__ __forceinline__ GateRows(const void* gate, long ts_, const Segment& s, int reverse, int head, int heads) {
        at = (const T*)gate + (reverse ? s.hi - kChunk : s.lo) * ts_ + head;
        ts = ts_;
        live = gate != nullptr && head < heads;
    }
    __device__ __forceinline__ T next(int rows, int reverse) {
        const BufRsrc from = whole_rsrc((const char*)at);
        const int lane = lane_id_again();
        const unsigned o = lane < (live ? rows : 0) ? times(reverse ? kChunk - 1 - lane : lane, ts * (long)sizeof(T)) : kNowhere;
        at += (reverse ? -kChunk : kChunk) * ts;
        if constexpr (sizeof(T) == 4) return __builtin_bit_cast(T, __builtin_amdgcn_raw_buffer_load_b32(from, (int)o, 0, 0));
        else return __builtin_bit_cast(T, __builtin_amdgcn_raw_buffer_load_b16(from, (int)o, 0, 0));
    }
};

// v of a column's four lanes (x, 0..3), summed in all of them
__device__ __forceinline__ float over_column(float v) {
    unsigned a = __builtin_bit_cast(unsigned, v);
    const u32x2 rows = __builtin_amdgcn_permlane16_swap(a, a, false, false);
    unsigned lo = rows[0], hi = rows[1];        // (a vector's element does not bit-cast: see frag_relu_bits)
    a = __builtin_bit_cast(unsigned, __builtin_bit_cast(float, lo) + __builtin_bit_cast(float, hi));
    const u32x2 halves = __builtin_amdgcn_permlane32_swap(a, a, false, false);
    lo = halves[0], hi = halves[1];
    return __builtin_bit_cast(float, lo) + __builtin_bit_cast(float, hi);
}

// Passes that do not wait for each other go into one launch, by blockIdx.z: of few tokens none fills the GPU (the gradient of 320 tokens and 8
// heads of 64: 39 -> 29 us; of 4 x 4096 and 16 of 128: 459 -> 410).  One alone is 2% faster when it need not look which it is.
template <class A, int N>
struct Calls {
    A call[N];
    __device__ __forceinline__ const A& mine() const { return call[N == 1 ? 0 : blockIdx.z]; }
};

// What a segment adds to the state, and the product of its gates.  A sweep without scores and outputs: 16384 tokens of 16 heads of 128 in bf16
// 34 us, 134 MB of keys and values and 38 MB of states at 5.1 TB/s.
template <class T, int D, int N>
__global__ void __launch_bounds__((Tile<T, D>::kThreads), (Tile<T, D>::kOccupancy)) recurrence_state_kernel(Calls<StateArgs, N> calls) {
    const StateArgs& p = calls.mine();
    typedef Tile<T, D> Ti;
    extern __shared__ __align__(16) char lds[];
    char* tb = lds;
    char* tc = tb + Ti::kBytes;
    Gates* gates = (Gates*)(tc + Ti::kBytes);
    unsigned* tops = (unsigned*)(gates + 2 * Ti::kHeads);           // [2][waves][heads][3]

    const Segment seg = find_segment(p.layout, blockIdx.x);
    if (!seg.live || seg.index == (p.reverse ? 0 : seg.count - 1)) return;     // nothing comes after it
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = lane_id();
    const int head0 = blockIdx.y * Ti::kHeads, mine = wave / Ti::kWavesPerHead, head = head0 + mine;
    const int slice = wave % Ti::kWavesPerHead * kSlice;
    const long len = seg.hi - seg.lo;
    const int chunks = (int)((len + kChunk - 1) / kChunk), steps = chunks * p.gb;

    State<T, D> state;
    state.clear();
    double exponent = 0.0;          // (a segment may have thousands of chunks, whose equal small exponents add up in fp32 with a drift)
    float unit = 1.0f, bound_s = 0.0f;
    typename Ti::Regs rb, rc;
    const int gate_wave = Ti::kWaves - 1 - wave;        // the last waves have the fewest scores to compute
    GateRows<T> gate_rows(p.gate, p.gate_ts, seg, p.reverse, head0 + gate_wave, p.heads);
    T g = (T)0.0f;
    double base = 0.0;              // of the head whose gates this wave sums
    const int heads = p.heads - head0;
    const long chunk = p.reverse ? -kChunk : kChunk;
    const char* pb = Ti::start(p.b, seg, p.reverse, head0 * p.gb);
    const char* pc = Ti::start(p.c, seg, p.reverse, head0 * p.gb);
    auto fetch = [&](long u, int sub) {         // the tiles of rows u.. and of the sub-th of the heads of (b, c); pb, pc: their first ones'
        const int rows = (int)min(len - u, (long)kChunk), t = Ti::thread(wave);
        Ti::load(rb, pb + sub * p.b.hs, p.b, p.reverse, p.gb, rows, heads, t);
        Ti::load(rc, pc + sub * p.c.hs, p.c, p.reverse, p.gb, rows, heads, t);
        if (sub + 1 == p.gb) {
            pb += chunk * p.b.ts;
            pc += chunk * p.c.ts;
        }
    };
    // gates run a chunk ahead of the tiles: they are summed by a wave while the others multiply
    auto gates_of = [&](long u) {
        if (gate_wave < Ti::kHeads && u < len) {
            run_gates<!Ti::kNormalise>(gates + (u / kChunk & 1) * Ti::kHeads + gate_wave, (float)g, p.reverse, 1.0f, p.weight_scale, Ti::kNormalise, base);
            g = gate_rows.next((int)min(len - u - kChunk, (long)kChunk), p.reverse);
        }
    };
    if (gate_wave < Ti::kHeads) g = gate_rows.next((int)min(len, (long)kChunk), p.reverse);
    fetch(0, 0);
    gates_of(0);
    __syncthreads();
    int sub = 0, next_sub = 0;
    long first = 0;
    for (int it = 0; it < steps; ++it, first += next_sub == 0 ? kChunk : 0, sub = next_sub) {
        unsigned* top = tops + (it & 1) * 3 * Ti::kWaves * Ti::kHeads;
        const int t = Ti::thread(wave);
        Ti::store(rb, tb, p.b.relu, t);
        const unsigned mc = Ti::store(rc, tc, p.c.relu, t);
        if constexpr (Ti::kNormalise) leave_top<Ti>(top + 2, mc);
        __syncthreads();
        if (it + 1 < steps) {
            next_sub = sub + 1 == p.gb ? 0 : sub + 1;
            fetch(first + (next_sub == 0 ? kChunk : 0), next_sub);
        }
        const Gates& gt = gates[(first / kChunk & 1) * Ti::kHeads + mine];
        if (sub == 0) gates_of(first + kChunk);
        float factor = 1.0f;
        if constexpr (Ti::kNormalise) {
            const float bound = tile_top<Ti>(top + 2, mine) * fabsf(p.weight_scale) * gt.grow;
            bound_s = (sub == 0 ? bound_s * gt.total : bound_s) + (float)kChunk * 65504.0f * bound;
            const float fresh = unit_of(bound, bound_s, unit);
            factor = fresh / unit;
            unit = fresh;
        }
        if (sub == 0) {
            factor *= gt.total;
            exponent += (double)gt.exponent;
            if constexpr (!Ti::kNormalise) unit = gt.unit;
        }
        if (factor != 1.0f) state.scale(factor);
        const int again = lane_id_again(), x = again & 15, q = again >> 4;
        typename Ti::Vec vt[Ti::kTokenSteps];
#pragma unroll
        for (int st = 0; st < Ti::kTokenSteps; ++st) vt[st] = Ti::value_operand(tc + mine * Ti::kHeadBytes, slice, st, x, q);
        state.add(tb + mine * Ti::kHeadBytes, vt, gt.weight, unit);
        __syncthreads();
    }
    if (head >= p.heads) return;
    const long at = (long)seg.slot * p.heads + head;
    state.write(p.own + at * (D * D), slice, p.rs, Ti::kNormalise ? 1.0f / unit : unit);
    if (lane == 0 && slice == 0) p.decay[at] = __builtin_amdgcn_exp2f((float)exponent);
}

// own[slot] (what a segment adds) becomes the state that the segment starts from, in the order of the scan.  Eight segments are read
// ahead: their loads hang on nothing.  CROSS, with `others` (the same of the scan in the opposite order, joined before): crossing[slot, head, workgroup]
// becomes the part of <own, others> at the border where a segment starts here and the one before it (in this order) started there, what the
// gates' gradient is summed up from.  36 segments of 16 heads of 128: 10 us, 75 MB at 7 TB/s out of the memory-side cache; small states wait
// for a chain of count / 8 loads (7 us at 32 segments; 12 or 16 ahead measured the same).
template <bool CROSS>
__global__ void __launch_bounds__(kThreads) recurrence_join_kernel(float* own, const float* decay, const float* first, Layout layout, int heads,
                                                                   int size, int reverse, const float* others, float* crossing) {
    constexpr int kAhead = 8;
    __shared__ float part[kAhead][kThreads / 64];
    const int b = blockIdx.x / heads, h = blockIdx.x % heads;
    const int e = (blockIdx.y * kThreads + threadIdx.x) * 4;
    const bool mine = e < size;
    const long slot0 = first_slot(layout, b);
    const long from = sequence_start(layout, b), to = max(from, sequence_start(layout, b + 1));
    const int count = (int)min(max(1L, (to - from + layout.segment - 1) / layout.segment), layout.slots - slot0);
    f32x4 run = {0, 0, 0, 0};
    if (mine && first != nullptr) run = *(const f32x4*)(first + ((long)b * heads + h) * size + e);
    for (int i0 = 0; i0 < count; i0 += kAhead) {
        f32x4 add[kAhead], other[kAhead];
        float keep[kAhead];
        static_for<0, kAhead>([&](auto i_) {
            constexpr int i = decltype(i_)::value;
            add[i] = other[i] = f32x4{0, 0, 0, 0};
            keep[i] = 0.0f;
            const int k = i0 + i;
            if (mine && k + 1 < count) {            // (nothing was summed for the last one)
                const long at = (slot0 + (reverse ? count - 1 - k : k)) * heads + h;
                add[i] = *(const f32x4*)(own + at * size + e);
                keep[i] = decay[at];
            }
            if (CROSS && mine && k > 0 && k < count)
                other[i] = *(const f32x4*)(others + ((slot0 + (reverse ? count - k : k - 1)) * heads + h) * size + e);
        });
        static_for<0, kAhead>([&](auto i_) {
            constexpr int i = decltype(i_)::value;
            const int k = i0 + i;
            if (k < count) {
                const long at = (slot0 + (reverse ? count - 1 - k : k)) * heads + h;
                if (mine) *(f32x4*)(own + at * size + e) = run;
                if constexpr (CROSS) {
                    const float dot = running_sum((run[0] * other[i][0] + run[1] * other[i][1]) + (run[2] * other[i][2] + run[3] * other[i][3]));
                    if (lane_id() == 63) part[i][threadIdx.x >> 6] = dot;
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) run[r] = fmaf(keep[i], run[r], add[i][r]);
            }
        });
        if constexpr (CROSS) {
            __syncthreads();
            const int k = i0 + (int)threadIdx.x;
            if (threadIdx.x < kAhead && k < count)
                crossing[((slot0 + (reverse ? count - 1 - k : k)) * heads + h) * gridDim.y + blockIdx.y] =
                    (part[threadIdx.x][0] + part[threadIdx.x][1]) + (part[threadIdx.x][2] + part[threadIdx.x][3]);
            __syncthreads();
        }
    }
}

template <class F>
__device__ __forceinline__ F load_through(BufRsrc r, unsigned off, unsigned scalar) {
    if constexpr (sizeof(F) == 8) return __builtin_bit_cast(F, __builtin_amdgcn_raw_buffer_load_b64(r, (int)off, (int)scalar, 0));
    else return __builtin_bit_cast(F, __builtin_amdgcn_raw_buffer_load_b128(r, (int)off, (int)scalar, 0));
}
// One of the scan's passes over a segment.  The tiles of the next chunk are on their way while this one's scores, outputs and state are
// computed; a wave has 16 output channels, so that the state (d rows of them) stays in its registers, and where four or more waves make a
// head each computes its share of the scores and all meet in LDS.
// 16384 tokens of 16 heads of 128 in bf16: 92 us (273 MB: 3.0 TB/s), with the masks and dot products 98.  No one unit is at its limit: of the cycles
// in which a compute unit holds waves the vector ALU is busy 57 % (some 690 instructions a wave and chunk), the matrix pipe 40 % (119), LDS 37 %; a
// wave spends 41 % of its time waiting for its turn to issue and 34 % for memory, LDS or a barrier.  The loop with nothing but its loads, LDS traffic
// and barriers takes 42 us.
// MASKED: out is masked and measured against m (p.m, p.dots).  GROUP: there are several heads of a, or of (b, c), to a state head.
template <class T, int D, bool MASKED, bool GROUP, int N>
__global__ void __launch_bounds__((Tile<T, D>::kThreads), (MASKED && Tile<T, D>::kWide16 ? 2 : Tile<T, D>::kOccupancy)) recurrence_sweep_kernel(Calls<SweepArgs, N> calls) {
    const SweepArgs& p = calls.mine();
    typedef Tile<T, D> Ti;
    typedef typename Ti::Vec Vec;
    typedef typename Ti::Op Op;
    typedef typename Ti::Frag Frag;
    typedef typename Ti::Tr Tr;
    constexpr int kThreads = Ti::kThreads;
    const int ga = GROUP ? p.ga : 1, gb = GROUP ? p.gb : 1, group = max(ga, gb);
    extern __shared__ __align__(16) char lds[];
    char* ta = lds;
    char* tb = ta + Ti::kBytes;
    char* tc = tb + Ti::kBytes;
    Gates* gates = (Gates*)(tc + Ti::kBytes);
    unsigned* tops = (unsigned*)(gates + 2 * Ti::kHeads);           // [2][waves][heads][3]
    float* dots = (float*)(tops + 6 * Ti::kWaves * Ti::kHeads);              // [waves][64]
    char* scores = (char*)(dots + kChunk * Ti::kWaves);

    const Segment seg = find_segment(p.layout, blockIdx.x);
    if (!seg.live) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int head0 = blockIdx.y * Ti::kHeads, mine = wave / Ti::kWavesPerHead, head = head0 + mine;
    const int slice = wave % Ti::kWavesPerHead * kSlice;
    const bool live = head < p.heads;
    const long len = seg.hi - seg.lo;
    const int chunks = (int)((len + kChunk - 1) / kChunk), steps = chunks * group;

    // (the upper halves of the steps of blocks 0 and 2 are above the diagonal, and stay zero)
    if constexpr (Ti::kShare)
        for (int i = threadIdx.x * 16; i < Ti::kScoreBytes; i += kThreads * 16) *(u32x4*)(scores + i) = u32x4{0, 0, 0, 0};
    State<T, D> state;
    if (live && p.start != nullptr) state.read(p.start + ((long)seg.slot * p.heads + head) * (D * D), slice, p.rs);
    else if (live && p.first != nullptr) state.read(p.first + ((long)seg.sequence * p.heads + head) * (D * D), slice, p.rs);
    else state.clear();
    float unit = 1.0f, bound_s = 0.0f, at = 0.0f, bt = 0.0f, ct = 0.0f;
    if constexpr (Ti::kNormalise) bound_s = state.top();

    typename Ti::Regs ra, rb, rc;
    const int gate_wave = Ti::kWaves - 1 - wave;        // the last waves have the fewest scores to compute
    GateRows<T> gate_rows(p.gate, p.gate_ts, seg, p.reverse, head0 + gate_wave, p.heads);
    T g = (T)0.0f;
    double base = 0.0;              // of the head whose gates this wave sums
    const int heads = p.heads - head0;
    const long chunk = p.reverse ? -kChunk : kChunk;
    const char* pa = Ti::start(p.a, seg, p.reverse, head0 * ga);
    const char* pb = Ti::start(p.b, seg, p.reverse, head0 * gb);
    const char* pc = Ti::start(p.c, seg, p.reverse, head0 * gb);
    auto fetch = [&](long u, int sub) {         // the tiles of rows u.. that the sub-th step of a chunk needs anew
        const int rows = (int)min(len - u, (long)kChunk), t = Ti::thread(wave);
        if (sub == 0 || ga > 1) Ti::load(ra, pa + (ga > 1 ? sub : 0) * p.a.hs, p.a, p.reverse, ga, rows, heads, t);
        if (sub == 0 || gb > 1) {
            Ti::load(rb, pb + (gb > 1 ? sub : 0) * p.b.hs, p.b, p.reverse, gb, rows, heads, t);
            Ti::load(rc, pc + (gb > 1 ? sub : 0) * p.c.hs, p.c, p.reverse, gb, rows, heads, t);
        }
        if (sub + 1 == group) {
            pa += chunk * p.a.ts;
            pb += chunk * p.b.ts;
            pc += chunk * p.c.ts;
        }
    };
    // rows 16i + x of out (and of what it is masked with) in the same way; a chunk's last 16 rows are its first ones from the end
    char* po = p.out + (p.reverse ? seg.hi - kChunk : seg.lo) * p.out_ts + (long)head * ga * p.out_hs + slice * (int)sizeof(T);
    const char* pm = MASKED ? Ti::start(p.m, seg, p.reverse, head * ga) + slice * (int)sizeof(T) : nullptr;
    // gates run a chunk ahead of the tiles: they are summed by a wave while the others multiply
    auto gates_of = [&](long u) {
        if (gate_wave < Ti::kHeads && u < len) {
            run_gates<!Ti::kNormalise>(gates + (u / kChunk & 1) * Ti::kHeads + gate_wave, (float)g, p.reverse, p.in_scale, p.weight_scale, Ti::kNormalise, base);
            g = gate_rows.next((int)min(len - u - kChunk, (long)kChunk), p.reverse);
        }
    };
    if (gate_wave < Ti::kHeads) g = gate_rows.next((int)min(len, (long)kChunk), p.reverse);
    if (steps > 0) fetch(0, 0);
    gates_of(0);
    f32x4 o[4];
    const bool hands_out = p.last != nullptr && seg.index == (p.reverse ? 0 : seg.count - 1);
    __syncthreads();
    int sub = 0, next_sub = 0;
    long first = 0;
    for (int it = 0; it < steps; ++it, first += next_sub == 0 ? kChunk : 0, sub = next_sub) {
        const bool new_a = sub == 0 || ga > 1, new_b = sub == 0 || gb > 1;      // (one of ga, gb is 1)
        const bool begins = new_a, ends = gb == 1 || sub == group - 1;            // of an output's sum
        const bool feeds = ga == 1 || sub == group - 1;                           // the state
        unsigned* top = tops + (it & 1) * 3 * Ti::kWaves * Ti::kHeads;
        unsigned ma = 0, mb = 0, mc = 0;
        const int t = Ti::thread(wave);
        if (new_a) ma = Ti::store(ra, ta, p.a.relu, t);
        if (new_b) {
            mb = Ti::store(rb, tb, p.b.relu, t);
            mc = Ti::store(rc, tc, p.c.relu, t);
        }
        if constexpr (Ti::kNormalise) {
            leave_top<Ti>(top, ma);
            leave_top<Ti>(top + 1, mb);
            leave_top<Ti>(top + 2, mc);
        }
        __syncthreads();
        // (a lane's number, and the addresses that are made of it, anew for each part: see Tile::load)
        int lane = lane_id_again(), x = lane & 15, q = lane >> 4;
        const Gates& gt = gates[(first / kChunk & 1) * Ti::kHeads + mine];
        if (sub == 0) gates_of(first + kChunk);
        const char* ha = ta + mine * Ti::kHeadBytes;
        char* hb = tb + mine * Ti::kHeadBytes;
        char* hc = tc + mine * Ti::kHeadBytes;
        float fp = 1.0f;
        if constexpr (Ti::kNormalise) {
            if (new_a) at = tile_top<Ti>(top, mine);
            if (new_b) {
                bt = tile_top<Ti>(top + 1, mine);
                ct = tile_top<Ti>(top + 2, mine);
            }
            fp = normaliser(fabsf(p.score_scale) * (float)D * at * bt * gt.grow);
        }
        const float score_scale = p.score_scale * fp;
        // scores of rows 16i + x and keys 16j + 4q + r
        auto score = [&](int i, int j, const Op (&va)[Ti::kSteps], float (&w)[4]) {
            f32x4 d = {0, 0, 0, 0};
#pragma unroll
            for (int s = 0; s < Ti::kSteps; ++s) d = Ti::mma(d, Ti::row_operand(hb, 16 * j + x, s, q), va[s]);
            const float fi = gt.hi[16 * i + x], li = gt.lo[16 * i + x];
            const f32x4 fj = *(const f32x4*)(gt.hi + 16 * j + 4 * q), lj = *(const f32x4*)(gt.lo + 16 * j + 4 * q);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float e = __builtin_amdgcn_exp2f((fi - fj[r]) + (li - lj[r]));
                w[r] = j < i || 4 * q + r <= x ? d[r] * e * score_scale : 0.0f;
            }
        };
        if constexpr (Ti::kShare) {
            // blocks 0, 1, .. of the lower triangle's ten, row by row, are dealt to the head's waves
#pragma unroll
            for (int k = 0; k < (10 + Ti::kWavesPerHead - 1) / Ti::kWavesPerHead; ++k) {
                int n = wave % Ti::kWavesPerHead + Ti::kWavesPerHead * k;
                asm volatile("" : "+s"(n));     // (its addresses are not worth registers all through the loop)
                if (n < 10) {
                    const int i = n >= 6 ? 3 : (n >= 3 ? 2 : (n >= 1 ? 1 : 0)), j = n - i * (i + 1) / 2;
                    Op va[Ti::kSteps];
#pragma unroll
                    for (int s = 0; s < Ti::kSteps; ++s) va[s] = Ti::row_operand(ha, 16 * i + x, s, q);
                    float w[4];
                    score(i, j, va, w);
                    Ti::leave_scores(w, scores + Ti::score_step(i, j / Ti::kJoin) * 1024 + lane * 16 + (Ti::kJoin == 2 ? (j & 1) * 8 : 0));
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        // what the rows take from the state
        if (begins) {
            float fs = 1.0f;
            if constexpr (Ti::kNormalise) fs = normaliser(bound_s * unit);
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int s = 0; s < Ti::kSteps; ++s) {
                Op va[4], part[kParts<T>];
#pragma unroll
                for (int i = 0; i < 4; ++i) va[i] = Ti::row_operand(ha, 16 * i + x, s, q);
                state.operand(s, fs, part);
#pragma unroll
                for (int k = 0; k < kParts<T>; ++k)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[i] = Ti::mma(o[i], part[k], va[i]);
                __builtin_amdgcn_sched_barrier(0);      // (or all steps' operands are read ahead, into registers that are not there)
            }
            const float undo = Ti::kNormalise ? 1.0f / (fs * unit) : 1.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float f = gt.in[16 * i + x];
                if constexpr (Ti::kNormalise) f *= undo;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    o[i][r] *= f;
                    if constexpr (Ti::kNormalise) o[i][r] *= fp;        // (f * fp may be above fp32's range where their product with this is not)
                }
            }
        } else if constexpr (Ti::kNormalise) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) o[i][r] *= fp;
        }
        // What out is masked with is asked for before the next tiles: loads return in order.  (Asked for here, and not at once, the tiles do not
        // hold registers through the part above.)
        const int rows = (int)min(len - first, (long)kChunk);
        Frag mv[MASKED ? 4 : 1];
        if constexpr (MASKED) {
            if (ends && live) {
                const unsigned om = times(p.reverse ? 15 - x : x, p.m.ts) + 4 * q * (unsigned)sizeof(T);
                const BufRsrc from = whole_rsrc(pm + (ga > 1 ? sub : 0) * p.m.hs);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    mv[i] = load_through<Frag>(from, x < rows - 16 * i ? om : kNowhere, (p.reverse ? 3 - i : i) * 16 * (unsigned)p.m.ts);
                if (sub + 1 == group) pm += chunk * p.m.ts;
            }
        }
        if (it + 1 < steps) {
            next_sub = sub + 1 == group ? 0 : sub + 1;
            fetch(first + (next_sub == 0 ? kChunk : 0), next_sub);
        }
        // what they take from the chunk's own rows
        if constexpr (Ti::kShare) __syncthreads();
        lane = lane_id_again(), x = lane & 15, q = lane >> 4;
        Vec vt[Ti::kTokenSteps];
#pragma unroll
        for (int st = 0; st < Ti::kTokenSteps; ++st) vt[st] = Ti::value_operand(hc, slice, st, x, q);
        if constexpr (Ti::kShare) {
            static_for<0, 4>([&](auto i_) {
                constexpr int i = decltype(i_)::value;
#pragma unroll
                for (int st = 0; st <= i / Ti::kJoin; ++st)
#pragma unroll
                    for (int k = 0; k < kParts<T>; ++k)
                        o[i] = Tr::mma_vec(o[i], vt[st], *(const Vec*)(scores + (k * Ti::kScoreSteps + Ti::score_step(i, st)) * 1024 + lane * 16));
                __builtin_amdgcn_sched_barrier(0);
            });
        } else {
            static_for<0, 4>([&](auto i_) {
                constexpr int i = decltype(i_)::value;
                Op va[Ti::kSteps];
#pragma unroll
                for (int s = 0; s < Ti::kSteps; ++s) va[s] = Ti::row_operand(ha, 16 * i + x, s, q);
                static_for<0, i / Ti::kJoin + 1>([&](auto st_) {
                    constexpr int st = decltype(st_)::value;
                    float w[kChunk / 16][4];
                    static_for<0, Ti::kJoin>([&](auto j_) {
                        constexpr int half = decltype(j_)::value, j = st * Ti::kJoin + half;
                        if constexpr (j <= i) {
                            score(i, j, va, w[half]);
                        } else {
#pragma unroll
                            for (int r = 0; r < 4; ++r) w[half][r] = 0.0f;
                        }
                    });
                    float flat[Ti::kVec];
#pragma unroll
                    for (int e = 0; e < Ti::kVec; ++e) flat[e] = w[e / 4][e % 4];
                    Vec part[kParts<T>];
                    Ti::template split<kParts<T>>(flat, part);
#pragma unroll
                    for (int k = 0; k < kParts<T>; ++k) o[i] = Tr::mma_vec(o[i], vt[st], part[k]);
                    __builtin_amdgcn_sched_barrier(0);
                });
            });
        }
        if constexpr (Ti::kNormalise) {
            const float undo = 1.0f / fp;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) o[i][r] *= undo;
        }
        if (ends && live) {
            const BufRsrc to = whole_rsrc(po + (ga > 1 ? sub : 0) * p.out_hs);
            if (sub + 1 == group) po += chunk * p.out_ts;
            lane = lane_id_again(), x = lane & 15, q = lane >> 4;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (MASKED) {
                    float dot = 0.0f;
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float me = Tr::to_f32(mv[i][r]);      // (0 where there is no row)
                        if (p.m.relu && !(me > 0.0f)) o[i][r] = 0.0f;
                        dot = fmaf(me, o[i][r], dot);
                    }
                    dot = over_column(dot);
                    if (q == 0) dots[wave * kChunk + 16 * i + x] = dot;
                }
            }
            if constexpr (sizeof(T) == 2) {
                // two rows of blocks trade halves between neighbouring groups of 16 lanes: a lane then has 8 channels of one row, 16 bytes
#pragma unroll
                for (int i = 0; i < 4; i += 2) {
                    const u32x2 a = __builtin_bit_cast(u32x2, frag_from_f32<T>(o[i])), b = __builtin_bit_cast(u32x2, frag_from_f32<T>(o[i + 1]));
                    const u32x2 s0 = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
                    const u32x2 s1 = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
                    const int row = 16 * (i + (q & 1)) + x;
                    const unsigned off = times(p.reverse ? kChunk - 1 - row : row, p.out_ts) + 16 * (q >> 1);
                    buf_store16(to, row < rows ? off : kNowhere, u32x4{s0[0], s1[0], s0[1], s1[1]});
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int row = 16 * i + x;
                    const unsigned off = times(p.reverse ? kChunk - 1 - row : row, p.out_ts) + 16 * q;
                    buf_store16(to, row < rows ? off : kNowhere, __builtin_bit_cast(u32x4, o[i]));
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        // the state behind the chunk
        if (feeds) {
            float factor = 1.0f;
            if constexpr (Ti::kNormalise) {
                const float bound = ct * fabsf(p.weight_scale) * gt.grow;
                bound_s = (new_b && sub > 0 && gb > 1 ? bound_s : bound_s * gt.total) + (float)kChunk * bt * bound;
                const float fresh = unit_of(bound, bound_s, unit);
                factor = fresh / unit;
                unit = fresh;
            }
            const bool decays = gb == 1 || sub == 0;
            if (decays) factor *= gt.total;
            if constexpr (!Ti::kNormalise) unit = gt.unit;
            if (factor != 1.0f) state.scale(factor);
            state.add(hb, vt, gt.weight, unit);
        }
        __syncthreads();
        if constexpr (MASKED) {
            // a row's dot product from its head's waves (the next ones are left behind two more barriers, or one that this wave has to reach)
            lane = lane_id_again();
            if (ends && p.dots != nullptr && wave < Ti::kHeads && lane < rows && head0 + wave < p.heads) {
                float dot = 0.0f;
#pragma unroll
                for (int w = 0; w < Ti::kWavesPerHead; ++w) dot += dots[(wave * Ti::kWavesPerHead + w) * kChunk + lane];
                const int hd = (head0 + wave) * ga + (ga > 1 ? sub : 0);
                p.dots[Ti::token(seg, p.reverse, first + lane) * (p.heads * ga) + hd] = dot;
            }
        }
    }
    if (live && hands_out)
        state.write(p.last + ((long)seg.sequence * p.heads + head) * (D * D), slice, p.rs, Ti::kNormalise ? 1.0f / unit : unit);
}

// d log_gate of a segment's tokens and one head: from the segment's end, x_t = q_t . dq_t - k_t . dk_t summed up, on top of <dS, S> at
// that end: the parts that the join left, or, at the sequence's end, of what came in and what was handed out there.
template <class T>
__global__ void __launch_bounds__(kThreads) recurrence_gate_kernel(const float* q_dots, const float* k_dots, const float* crossing, int parts,
                                                                   const float* last, const float* d_last, T* d_gate, long d_gate_ts, Layout layout,
                                                                   int heads, int group, int size) {
    __shared__ double part[kThreads / 64];
    const Segment seg = find_segment(layout, blockIdx.x);
    if (!seg.live) return;
    const int h = blockIdx.y, wave = threadIdx.x >> 6, lane = lane_id();
    double sum = 0.0;
    if (seg.index < seg.count - 1) {
        if ((int)threadIdx.x < parts) sum = (double)crossing[((long)seg.slot * heads + h) * parts + threadIdx.x];
    } else if (last != nullptr && d_last != nullptr) {
        const float* sp = last + ((long)seg.sequence * heads + h) * size;
        const float* dp = d_last + ((long)seg.sequence * heads + h) * size;
        for (int e = threadIdx.x * 4; e < size; e += kThreads * 4) {
            const f32x4 a = *(const f32x4*)(sp + e), b = *(const f32x4*)(dp + e);
#pragma unroll
            for (int r = 0; r < 4; ++r) sum += (double)a[r] * (double)b[r];
        }
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    if (lane == 0) part[wave] = sum;
    __syncthreads();
    double above = part[0] + part[1] + part[2] + part[3];
    const long len = seg.hi - seg.lo;
    for (long u0 = 0; u0 < len; u0 += kThreads) {           // rows from the end
        const long u = u0 + threadIdx.x, t = seg.hi - 1 - u;
        double x = 0.0;
        if (u < len) {
            for (int g = 0; g < group; ++g) x += (double)q_dots[(t * heads + h) * group + g];
            x -= (double)k_dots[t * heads + h];
        }
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const double up = __shfl_up(x, d);
            if (lane >= d) x += up;
        }
        __syncthreads();
        if (lane == 63) part[wave] = x;
        __syncthreads();
        double before = above;
        for (int w = 0; w < wave; ++w) before += part[w];
        if (u < len) d_gate[t * d_gate_ts + h] = (T)(float)(before + x);
        above += part[0] + part[1] + part[2] + part[3];
    }
}

struct StepArgs {
    Heads q, k, v;
    const void* gate;
    long gate_ts;
    const float* state;
    float* fresh;
    char* out;
    long out_ts, out_hs;
    long units;                     // sequences * heads
    int heads, group;
    float scale;
};

// One token a sequence: the state is read once and written once, which is what there is to do (192 sequences of 16 heads of 128: 407 MB in
// 81 us, 5.0 TB/s; one sequence 4 us).  A workgroup has 32 columns of a
// state (16 for heads of 16): eight lanes a row of them, 16 bytes each, so a thread holds d/32 rows; heads of 16 go four to a workgroup.
template <class T, int D>
__global__ void __launch_bounds__(kThreads) recurrence_step_kernel(StepArgs p) {
    typedef Traits<T> Tr;
    constexpr int kCols = D < 32 ? D : 32, kLanes = kCols / 4, kGroups = kThreads / kLanes;
    constexpr int kUnits = D < kGroups ? kGroups / D : 1;           // states of a workgroup
    constexpr int kRowLanes = kGroups / kUnits, kRows = D / kRowLanes;
    constexpr int kSlices = D / kCols;
    __shared__ float part[4][kCols];
    const int lane = threadIdx.x % kLanes, group = threadIdx.x / kLanes;
    const long unit = (long)(blockIdx.x / kSlices) * kUnits + group / kRowLanes;
    const int row0 = group % kRowLanes, col = blockIdx.x % kSlices * kCols + lane * 4;
    const bool live = unit < p.units;
    const long b = live ? unit / p.heads : 0;
    const int h = live ? (int)(unit % p.heads) : 0;
    f32x4 s[kRows];
    const float* from = p.state == nullptr ? nullptr : p.state + (b * p.heads + h) * (D * D) + col;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        s[i] = f32x4{0, 0, 0, 0};
        if (live && from != nullptr) s[i] = *(const f32x4*)(from + (row0 + i * kRowLanes) * D);
    }
    const T* kp = (const T*)(p.k.p + b * p.k.ts + h * p.k.hs);
    const f32x4 v = frag_to_f32<T>(load_frag<T>((const T*)(p.v.p + b * p.v.ts + h * p.v.hs) + col));
    float keep = 1.0f;
    if (p.gate != nullptr) {
        const float g = (float)((const T*)p.gate)[b * p.gate_ts + h];
        keep = expf(g);
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        float k = Tr::to_f32(kp[row0 + i * kRowLanes]);
        if (p.k.relu) k = k <= 0.0f ? 0.0f : k;       // (a NaN stays one, as in the scan)
#pragma unroll
        for (int r = 0; r < 4; ++r) s[i][r] = fmaf(k, v[r], keep * s[i][r]);
        if (live) *(f32x4*)(p.fresh + (b * p.heads + h) * (D * D) + (row0 + i * kRowLanes) * D + col) = s[i];
    }
    for (int g = 0; g < p.group; ++g) {
        const T* qp = (const T*)(p.q.p + b * p.q.ts + (h * p.group + g) * p.q.hs);
        f32x4 o = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            float q = Tr::to_f32(qp[row0 + i * kRowLanes]);
            if (p.q.relu) q = q <= 0.0f ? 0.0f : q;
#pragma unroll
            for (int r = 0; r < 4; ++r) o[r] = fmaf(q, s[i][r], o[r]);
        }
#pragma unroll
        for (int d = kLanes; d < 64; d *= 2)
#pragma unroll
            for (int r = 0; r < 4; ++r) o[r] += __shfl_xor(o[r], d);
        T* out = (T*)(p.out + b * p.out_ts + (h * p.group + g) * p.out_hs) + col;
        if constexpr (kRowLanes * kLanes <= 64) {
            if (live && row0 == 0) {
#pragma unroll
                for (int r = 0; r < 4; ++r) o[r] *= p.scale;
                store_frag<T>(out, frag_from_f32<T>(o));
            }
        } else {
            const int wave = threadIdx.x >> 6;
            if ((threadIdx.x & 63) < kLanes) *(f32x4*)&part[wave][lane * 4] = o;
            __syncthreads();
            if (threadIdx.x < kLanes && live) {
#pragma unroll
                for (int r = 0; r < 4; ++r) o[r] = ((part[0][lane * 4 + r] + part[1][lane * 4 + r]) + (part[2][lane * 4 + r] + part[3][lane * 4 + r])) * p.scale;
                store_frag<T>(out, frag_from_f32<T>(o));
            }
            __syncthreads();
        }
    }
}

// ------------------------------------------------------------------------------------------------ host side
template <class T, int D>
constexpr int tile_lds(int tiles) { return tiles * Tile<T, D>::kBytes + 2 * Tile<T, D>::kHeads * (int)sizeof(Gates) + 6 * Tile<T, D>::kWaves * Tile<T, D>::kHeads * 4; }
template <class T, int D>
constexpr int sweep_lds() { return tile_lds<T, D>(3) + kChunk * Tile<T, D>::kWaves * 4 + Tile<T, D>::kScoreBytes; }

// LDS above the 64 KB that a kernel may ask for by itself is granted once a kernel and device
template <class K>
hipError_t allow_lds(K kernel, int bytes, unsigned long long* done) {
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    const unsigned long long bit = 1ull << (dev & 63);
    if (bytes <= 65536 || (__atomic_load_n(done, __ATOMIC_ACQUIRE) & bit)) return hipSuccess;
    e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == hipSuccess) __atomic_fetch_or(done, bit, __ATOMIC_RELEASE);
    return e;
}

template <class T, int D, int N>
hipError_t launch_state(const Calls<StateArgs, N>& c, hipStream_t stream) {
    static unsigned long long done = 0;
    constexpr int bytes = tile_lds<T, D>(2);
    hipError_t e = allow_lds(&recurrence_state_kernel<T, D, N>, bytes, &done);
    if (e != hipSuccess) return e;
    const StateArgs& a = c.call[0];
    const dim3 grid(a.layout.slots, (a.heads + Tile<T, D>::kHeads - 1) / Tile<T, D>::kHeads, N);
    hipLaunchKernelGGL((recurrence_state_kernel<T, D, N>), grid, dim3(Tile<T, D>::kThreads), bytes, stream, c);
    return hipGetLastError();
}

template <class T, int D, bool MASKED, bool GROUP, int N>
hipError_t launch_sweep_as(const Calls<SweepArgs, N>& c, hipStream_t stream) {
    static unsigned long long done = 0;
    constexpr int bytes = sweep_lds<T, D>();
    hipError_t e = allow_lds(&recurrence_sweep_kernel<T, D, MASKED, GROUP, N>, bytes, &done);
    if (e != hipSuccess) return e;
    const SweepArgs& a = c.call[0];
    const dim3 grid(a.layout.slots, (a.heads + Tile<T, D>::kHeads - 1) / Tile<T, D>::kHeads, N);
    hipLaunchKernelGGL((recurrence_sweep_kernel<T, D, MASKED, GROUP, N>), grid, dim3(Tile<T, D>::kThreads), bytes, stream, c);
    return hipGetLastError();
}

// (calls of one layout and group)
template <class T, int D, bool MASKED, int N>
hipError_t launch_sweep(const Calls<SweepArgs, N>& c, hipStream_t stream) {
    if (c.call[0].ga > 1 || c.call[0].gb > 1) return launch_sweep_as<T, D, MASKED, true>(c, stream);
    return launch_sweep_as<T, D, MASKED, false>(c, stream);
}

int join_groups(int size) { return (size / 4 + kThreads - 1) / kThreads; }

hipError_t launch_join(float* own, const float* decay, const float* first, const Layout& l, int heads, int size, int reverse, const float* others,
                       float* crossing, hipStream_t stream) {
    const dim3 grid(l.sequences * heads, join_groups(size));
    if (others != nullptr) hipLaunchKernelGGL(recurrence_join_kernel<true>, grid, dim3(kThreads), 0, stream, own, decay, first, l, heads, size, reverse, others, crossing);
    else hipLaunchKernelGGL(recurrence_join_kernel<false>, grid, dim3(kThreads), 0, stream, own, decay, first, l, heads, size, reverse, others, crossing);
    return hipGetLastError();
}

template <class T>
Heads heads_of(const RecurrenceRows& r, int relu) {
    return Heads{(const char*)r.p, r.ts * (long)sizeof(T), r.hs * (long)sizeof(T), relu};
}
// ... of an output: pointer and strides
#define MSLA_OUT(r) (char*)(r).p, (r).ts * (long)sizeof(T), (r).hs * (long)sizeof(T)


Layout layout_of(const RecurrenceCall& c) {
    return Layout{c.offsets, c.sequences, c.tokens, c.plan.segment, c.plan.slots};
}

#define MSLA_TRY(x)                         \
    do {                                    \
        const hipError_t e_ = (x);          \
        if (e_ != hipSuccess) return e_;    \
    } while (0)

template <class T, int D>
hipError_t forward_of(const RecurrenceCall& c, hipStream_t stream) {
    const Layout l = layout_of(c);
    const Heads q = heads_of<T>(c.q, c.rectify), k = heads_of<T>(c.k, c.rectify), v = heads_of<T>(c.v, 0);
    const float* start = nullptr;
    if (c.plan.cut) {
        float* own = (float*)c.ws;
        float* decay = (float*)(c.ws + c.plan.decay_at);
        MSLA_TRY((launch_state<T, D, 1>({{StateArgs{k, v, c.gate, c.gate_ts, own, decay, D, l, c.heads_kv, 1, 0, 1.0f}}}, stream)));
        MSLA_TRY(launch_join(own, decay, c.initial, l, c.heads_kv, D * D, 0, nullptr, nullptr, stream));
        start = own;
    }
    return launch_sweep<T, D, false, 1>({{SweepArgs{q, k, v, MSLA_OUT(c.out), Heads{nullptr, 0, 0, 0}, nullptr, c.gate, c.gate_ts, start, c.initial,
                                          c.final_state, D, l, c.heads_kv, c.heads_q / c.heads_kv, 1, 0, c.scale, c.scale, 1.0f}}}, stream);
}

template <class T, int D>
hipError_t backward_of(const RecurrenceCall& c, hipStream_t stream) {
    const Layout l = layout_of(c);
    const int group = c.heads_q / c.heads_kv;
    const Heads q = heads_of<T>(c.q, c.rectify), k = heads_of<T>(c.k, c.rectify), v = heads_of<T>(c.v, 0), d_o = heads_of<T>(c.d_out, 0);
    const Heads no = {nullptr, 0, 0, 0};
    float* s_own = nullptr;
    float* d_own = nullptr;
    float* crossing = (float*)(c.ws + c.plan.crossing_at);
    if (c.plan.cut) {
        s_own = (float*)c.ws;
        d_own = (float*)(c.ws + c.plan.d_states_at);
        float* decay = (float*)(c.ws + c.plan.decay_at);
        float* d_decay = (float*)(c.ws + c.plan.d_decay_at);
        MSLA_TRY((launch_state<T, D, 2>({{StateArgs{v, k, c.gate, c.gate_ts, s_own, decay, 1, l, c.heads_kv, 1, 0, 1.0f},
                                       StateArgs{d_o, q, c.gate, c.gate_ts, d_own, d_decay, 1, l, c.heads_kv, group, 1, c.scale}}}, stream)));
        MSLA_TRY(launch_join(s_own, decay, c.initial, l, c.heads_kv, D * D, 0, nullptr, nullptr, stream));
        MSLA_TRY(launch_join(d_own, d_decay, c.d_final, l, c.heads_kv, D * D, 1, c.d_gate ? s_own : nullptr, crossing, stream));
    }
    float* q_dots = c.d_gate ? (float*)(c.ws + c.plan.dots_at) : nullptr;
    float* k_dots = c.d_gate ? q_dots + c.tokens * c.heads_q : nullptr;
    float* last = c.d_gate && c.d_final ? (float*)(c.ws + c.plan.last_at) : nullptr;
    const Heads mq = c.d_gate || c.rectify ? q : no, mk = c.d_gate || c.rectify ? k : no;
    const SweepArgs d_q{d_o, v, k, MSLA_OUT(c.d_q), mq, q_dots, c.gate, c.gate_ts, s_own, c.initial, last, 1, l, c.heads_kv, group, 1, 0, c.scale, c.scale, 1.0f};
    const SweepArgs d_k{v, d_o, q, MSLA_OUT(c.d_k), mk, k_dots, c.gate, c.gate_ts, d_own, c.d_final, nullptr, 1, l, c.heads_kv, 1, group, 1, c.scale, 1.0f, c.scale};
    const SweepArgs d_v{k, q, d_o, MSLA_OUT(c.d_v), no, nullptr, c.gate, c.gate_ts, d_own, c.d_final, c.d_initial, D, l, c.heads_kv, 1, group, 1, c.scale, 1.0f, c.scale};
    if (mq.p != nullptr) {
        MSLA_TRY((launch_sweep<T, D, true, 2>({{d_q, d_k}}, stream)));
        MSLA_TRY((launch_sweep<T, D, false, 1>({{d_v}}, stream)));
    } else {
        MSLA_TRY((launch_sweep<T, D, false, 3>({{d_q, d_k, d_v}}, stream)));
    }
    if (c.d_gate) {
        hipLaunchKernelGGL((recurrence_gate_kernel<T>), dim3(l.slots, c.heads_kv), dim3(kThreads), 0, stream, q_dots, k_dots, crossing, join_groups(D * D), last, c.d_final, (T*)c.d_gate, c.d_gate_ts, l, c.heads_kv, group, D * D);
        MSLA_TRY(hipGetLastError());
    }
    return hipSuccess;
}

template <class T, int D>
hipError_t step_of(const RecurrenceCall& c, hipStream_t stream) {
    constexpr int kCols = D < 32 ? D : 32, kGroups = kThreads / (kCols / 4), kUnits = D < kGroups ? kGroups / D : 1;
    const long units = (long)c.sequences * c.heads_kv;
    const long blocks = (units + kUnits - 1) / kUnits * (D / kCols);
    hipLaunchKernelGGL((recurrence_step_kernel<T, D>), dim3((unsigned)blocks), dim3(kThreads), 0, stream,
                       StepArgs{heads_of<T>(c.q, c.rectify), heads_of<T>(c.k, c.rectify), heads_of<T>(c.v, 0), c.gate, c.gate_ts, c.initial,
                                c.final_state, MSLA_OUT(c.out), units, c.heads_kv, c.heads_q / c.heads_kv, c.scale});
    return hipGetLastError();
}

template <class T, int D>
hipError_t run_of(const RecurrenceCall& c, hipStream_t stream) {
    switch (c.what) {
        case 0: return forward_of<T, D>(c, stream);
        case 1: return backward_of<T, D>(c, stream);
        default: return step_of<T, D>(c, stream);
    }
}

template <class T>
hipError_t run_for(const RecurrenceCall& c, hipStream_t stream) {
    switch (c.head_dim) {
        case 16: return run_of<T, 16>(c, stream);
        case 32: return run_of<T, 32>(c, stream);
        case 64: return run_of<T, 64>(c, stream);
        case 128: return run_of<T, 128>(c, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace rec

hipError_t launch_recurrence(int dt, const RecurrenceCall& c, hipStream_t stream) {
    switch (dt) {
        case 0: return rec::run_for<float>(c, stream);
        case 1: return rec::run_for<_Float16>(c, stream);
        case 2: return rec::run_for<__bf16>(c, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace msla
