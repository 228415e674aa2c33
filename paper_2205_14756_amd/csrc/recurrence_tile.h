// What the kernels of the gated recurrence (k_recurrence.hip) share: where segments lie, how a chunk of 64 tokens enters LDS, the
// chunk's running gates, and operands of the matrix instructions out of both.
//
// A workgroup walks over the chunks of one segment; a wave owns 16 output channels of one head, so that its part of the state leaves room for
// three or four waves on a SIMD: this work is a mixture of matrix and vector instructions and LDS latency, and what hides one is another wave.
// A head of 128 is a workgroup of eight waves; workgroups of four hold one head of 64, two of 32 or four of 16.
//
// Which register holds what is chosen so that nothing is ever transposed: a result D of a 16x16 matrix instruction (lane (x, q): rows
// 4q + r, column x) is at once the next one's operand (lane (x, q): the contraction slots that q owns, of row or column x).
//   - scores come as b a^T, so lane (x, q) has query x and keys 4q + r of each block of 16: an operand over the keys;
//   - the state's rows (channels of the key) are dealt to the blocks so that two of them hold 8 neighbouring channels a lane, in the order
//     in which a row of queries is read from LDS 16 bytes a lane;
//   - operands over tokens out of token-major tiles are gathered by ds_read_b64_tr_b16 (4x16 blocks, any address a lane).
#pragma once
#include "msla_device.h"

namespace msla {
namespace rec {

constexpr int kChunk = 64;
constexpr int kSlice = 16;          // output channels of a wave

struct Heads {
    const char* p;
    long ts, hs;                    // bytes from a token, and a head, to the next (below 2^24, and at most 2^29)
    int relu;
};

struct Layout {
    const int* offsets;
    int sequences;
    long tokens;
    int segment;                    // tokens of a segment, a multiple of kChunk
    int slots;                      // segments of all sequences have distinct numbers below this
};

__device__ __forceinline__ long sequence_start(const Layout& l, int b) {
    if (l.offsets == nullptr) return l.tokens / l.sequences * b;
    const long at = l.offsets[b];
    return at < 0 ? 0 : (at > l.tokens ? l.tokens : at);
}

// Segment numbers: sequence b's begin at start(b) / segment + b, which leaves room for all of them (and for one where it is
// empty), so a workgroup finds its own without anyone counting lengths first.
__device__ __forceinline__ long first_slot(const Layout& l, int b) { return sequence_start(l, b) / l.segment + b; }

// (the same in all lanes, and known to be: addresses made of it are scalar)
__device__ __forceinline__ long uniform(long v) {
    return (long)((unsigned long)(unsigned)__builtin_amdgcn_readfirstlane((int)((unsigned long)v >> 32)) << 32 |
                  (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned long)v));
}

struct Segment {
    int sequence, index, count, slot;
    long lo, hi;                    // its tokens
    bool live;
};

__device__ __forceinline__ Segment find_segment(const Layout& l, int slot) {
    int lo = 0, hi = l.sequences - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (first_slot(l, mid) <= slot) lo = mid;
        else hi = mid - 1;
    }
    Segment s;
    lo = __builtin_amdgcn_readfirstlane(lo);
    s.sequence = lo;
    s.slot = slot;
    const long from = uniform(sequence_start(l, lo)), to = max(from, uniform(sequence_start(l, lo + 1)));
    s.index = slot - (int)first_slot(l, lo);
    s.count = max(1, (int)((to - from + l.segment - 1) / l.segment));
    s.live = s.index >= 0 && s.index < s.count;
    s.lo = from + (long)s.index * l.segment;
    s.hi = min(to, s.lo + l.segment);
    return s;
}

// Parts of an operand that is not an input (scores, the state on its way into an output, what is added to the state): as many as leave fp32's
// own precision, three in bf16 (2^-25 of the value), two in fp16 (2^-23).  Two in bf16 (2^-17) moved one output in 400 by a rounding, and
// 16384 tokens of 16 heads of 128 in 138 us instead of 148 (their gradient 380, 419).
template <class T> constexpr int kParts = sizeof(T) == 4 ? 1 : (std::is_same<T, __bf16>::value ? 3 : 2);

// A resource over all that a 32-bit offset reaches, and an offset outside of it.
constexpr unsigned kNowhere = 0xfffffff0u;
__device__ __forceinline__ BufRsrc whole_rsrc(const char* at) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(at), 0, (int)kNowhere, 0x00020000);
}

// a row's number, below 256, times a token's stride (a product of 24-bit factors issues four times as fast as one of 32)
__device__ __forceinline__ unsigned times(unsigned row, long ts) { return __umul24(row, (unsigned)ts); }

template <class T, int D>
struct Tile {
    typedef Traits<T> Tr;
    typedef typename Tr::Vec Vec;               // an operand over tokens
    typedef typename Tr::Frag Frag;
    static constexpr int kVec = Tr::kVec;
    static constexpr int kWaves = D == 128 ? 8 : 4, kThreads = 64 * kWaves;
    static constexpr int kWavesPerHead = D / kSlice;
    static constexpr int kHeads = kWaves / kWavesPerHead;       // heads of a workgroup
    // waves that a SIMD has room for by registers and LDS
    static constexpr int kOccupancy = sizeof(T) == 4 ? 2 : (D == 64 ? 3 : 4);
    // heads of 128 in fp16, whose normalisers need registers of their own
    static constexpr bool kWide16 = D == 128 && std::is_same<T, _Float16>::value;
    // an operand over channels: 16 bytes a lane, for heads of 16 in 16 bits 8 (16 channels make one of the smaller matrix instruction's)
    static constexpr int kOp = D == 16 ? 4 : kVec;
    typedef typename std::conditional<D == 16, Frag, Vec>::type Op;
    static constexpr int kStep = 4 * kOp;                       // channels of one matrix step (fp32: four instructions)
    static constexpr int kSteps = D / kStep;
    static constexpr int kBlocks = D / 16;                      // blocks of 16 key channels
    static constexpr int kJoinOp = kOp / 4;                     // results that make one operand over channels
    static constexpr int kTokenStep = 4 * kVec;                 // ... over tokens
    static constexpr int kTokenSteps = kChunk / kTokenStep;
    static constexpr int kJoin = kVec / 4;
    // rows 32 bytes apart modulo 128 (16 where they are 32 long): the rows that a read serves together, and the four of a gather, spread
    // over the banks
    static constexpr int kPitch = D * (int)sizeof(T) + (D * sizeof(T) == 32 ? 16 : 32);
    static constexpr int kHeadBytes = kChunk * kPitch;
    static constexpr int kBytes = kHeads * kHeadBytes;
    static constexpr int kPerRow = kHeads * (D / kVec);         // 16-byte pieces of a tile's row
    static constexpr int kPieces = kChunk * kPerRow / kThreads;     // of a thread
    static_assert(kChunk * kPerRow % kThreads == 0 && kThreads % kPerRow == 0, "whole rows a pass");
    // Scores of a head are the same for its waves: where there are four or eight, each computes its share of them and leaves its parts in LDS
    // as operands, 1 KB a matrix step and part; where there are two (or one), each has them all in registers.
    static constexpr bool kShare = kWavesPerHead >= 4;
    static constexpr int kScoreSteps = kJoin == 2 ? 6 : 10;     // steps of the lower triangle's four rows of blocks
    static constexpr int kScoreBytes = kShare ? kScoreSteps * 1024 * kParts<T> : 0;
    static __device__ __forceinline__ constexpr int score_step(int i, int st) { return kJoin == 2 ? (i < 2 ? i : 2 * i - 2) + st : i * (i + 1) / 2 + st; }
    static constexpr bool kNormalise = std::is_same<T, _Float16>::value;

    struct Regs { u32x4 v[kPieces]; };

    static __device__ __forceinline__ f32x4 mma(f32x4 c, const Op& a, const Op& b) {
        if constexpr (D == 16) return Tr::mma16(c, a, b);
        else return Tr::mma_vec(c, a, b);
    }

    // key channel of row m of block `blk`: see the top of the file
    static __device__ __forceinline__ int channel(int blk, int m) {
        return kJoinOp == 2 ? 32 * (blk >> 1) + 8 * (m >> 2) + 4 * (blk & 1) + (m & 3) : 16 * blk + m;
    }

    static constexpr int kRowStep = kThreads / kPerRow;         // rows between a thread's pieces

    static __device__ __forceinline__ long token(const Segment& s, int reverse, long u) { return reverse ? s.hi - 1 - u : s.lo + u; }

    // A thread's pieces of a tile: rows row(t) + i * kRowStep, through a buffer resource at the tile's lowest address: one 32-bit offset a
    // thread and tile, a scalar one a piece.  (The host refuses strides whose sum, group of query heads included, does not stay below kNowhere.)  The thread's number t is made anew for each
    // tile, and the offset of it: kept over the loop, they cost registers that are not there, and what is spilled here is waited for among
    // the loads in flight.
    static __device__ __forceinline__ int row(int t) { return t / kPerRow; }
    static __device__ __forceinline__ int head_of(int t) { return t % kPerRow / (D / kVec); }
    static __device__ __forceinline__ int thread(int wave) { return 64 * wave + lane_id_again(); }
    // the lowest address of the segment's first chunk (from the end: of the last tokens' chunk) and of a head
    static __device__ __forceinline__ const char* start(const Heads& h, const Segment& s, int reverse, int head) {
        return h.p + (reverse ? s.hi - kChunk : s.lo) * h.ts + head * h.hs;
    }
    // Rows above `rows` are not the segment's, heads above `heads` nobody's: zero, and not read, by the resource's range check, which leaves no
    // branch around a load and nothing to wait for.
    static __device__ __forceinline__ void load(Regs& r, const char* at, const Heads& h, int reverse, int per, int rows, int heads, int t) {
        const BufRsrc from = whole_rsrc(at);
        const unsigned step = (unsigned)kRowStep * (unsigned)h.ts;
        unsigned off = times((unsigned)(reverse ? kRowStep - 1 - row(t) : row(t)), h.ts) + t % (D / kVec) * 16u;
        if (kHeads > 1) off += (unsigned)(head_of(t) * per) * (unsigned)h.hs;
        if (kHeads > 1 && head_of(t) >= heads) off = kNowhere;
#pragma unroll
        for (int i = 0; i < kPieces; ++i)
            r.v[i] = buf_load16(from, row(t) < rows - i * kRowStep ? off : kNowhere, (int)((reverse ? kPieces - 1 - i : i) * step));
    }

    // max(x, 0) of 16 bytes, and a NaN stays one, of either sign.  On the bits: a signed maximum with 0 takes what is negative to 0, NaNs with a sign
    // among it, and those are what lies above -inf as an unsigned number; 0 less that distance is a NaN again.
    static __device__ __forceinline__ u32x4 rectified(u32x4 v) {
        typedef typename std::conditional<sizeof(T) == 2, short, int>::type I;
        typedef typename std::conditional<sizeof(T) == 2, unsigned short, unsigned>::type U;
        typedef I Signed __attribute__((ext_vector_type(kVec)));
        typedef U Unsigned __attribute__((ext_vector_type(kVec)));
        const Unsigned infinite = (Unsigned)(U)(std::is_same<T, float>::value ? 0xff800000u : (kNormalise ? 0xfc00u : 0xff80u));
        const Unsigned positive = __builtin_bit_cast(Unsigned, __builtin_elementwise_max(__builtin_bit_cast(Signed, v), (Signed)(I)0));
        return __builtin_bit_cast(u32x4, positive - __builtin_elementwise_sub_sat(__builtin_bit_cast(Unsigned, v), infinite));
    }

    // into LDS, rectified where asked; returns the largest bit pattern of a finite magnitude of this lane's pieces (fp16 alone; one that is not
    // finite bounds nothing, and would take the rest of its head along)
    static __device__ __forceinline__ unsigned store(Regs& r, char* tile, int relu, int t) {
        unsigned top = 0;
        if (relu) {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) r.v[i] = rectified(r.v[i]);
        }
        char* at = tile + head_of(t) * kHeadBytes + row(t) * kPitch + t % (D / kVec) * 16;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            if constexpr (kNormalise) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const unsigned lo = r.v[i][j] & 0x7fffu, hi = (r.v[i][j] >> 16) & 0x7fffu;
                    top = max(top, max(lo < 0x7c00u ? lo : 0u, hi < 0x7c00u ? hi : 0u));
                }
            }
            *(u32x4*)(at + i * kRowStep * kPitch) = r.v[i];
        }
        return top;
    }

    // operand over channels: row `row`, channels of step s
    static __device__ __forceinline__ Op row_operand(const char* tile, int row, int s, int q) {
        return *(const Op*)(tile + row * kPitch + (s * kStep + kOp * q) * (int)sizeof(T));
    }

    // Operand over tokens, token slots of step s (16-bit: 32s + 4q + r and 16 further on; fp32: 16s + 4q + r): column x of the 16 channels
    // that start at `at` (bytes into a row), four of them every `apart` bytes.
    static __device__ __forceinline__ Vec gather(char* tile, int at, int apart, int s, int x, int q) {
        if constexpr (sizeof(T) == 2) {
            typedef __attribute__((address_space(3))) i16x4* LdsPtr;
            char* from = tile + (32 * s + 4 * q + (x >> 2)) * kPitch + at + apart * (x & 3);
            const i16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)from);
            const i16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)(from + 16 * kPitch));
            typedef short i16x8 __attribute__((ext_vector_type(8)));
            return __builtin_bit_cast(Vec, i16x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]});
        } else {
            Vec v;
#pragma unroll
            for (int r = 0; r < 4; ++r) v[r] = *(const float*)(tile + (16 * s + 4 * q + r) * kPitch + at + x * 4);
            return v;
        }
    }
    // ... rows of block `blk` of the state; the wave's own output channels
    static __device__ __forceinline__ Vec key_operand(char* tile, int blk, int s, int x, int q) {
        if constexpr (kJoinOp == 2) return gather(tile, 64 * (blk >> 1) + 8 * (blk & 1), 16, s, x, q);
        else return gather(tile, 16 * blk * (int)sizeof(T), 8, s, x, q);
    }
    static __device__ __forceinline__ Vec value_operand(char* tile, int slice, int s, int x, int q) {
        return gather(tile, slice * (int)sizeof(T), 8, s, x, q);
    }

    // four scores as operands' parts: half a step of them (fp32: a whole one) at `to`
    static __device__ __forceinline__ void leave_scores(const float (&w)[4], char* to) {
        Frag part[kParts<T>];
        split<kParts<T>>(w, part);
#pragma unroll
        for (int p = 0; p < kParts<T>; ++p) store_frag<T>(to + p * kScoreSteps * 1024, part[p]);
    }

    // v in PARTS parts of the storage type, each what the ones before left.  Pairs at a time: a rounded pair is one register, and is taken apart
    // again by a shift and a mask (bf16) instead of being rounded twice.
    template <int PARTS, class V, int N>
    static __device__ __forceinline__ void split(const float (&v)[N], V (&part)[PARTS]) {
        if constexpr (sizeof(T) == 4) {
            static_assert(PARTS == 1, "fp32 is whole");
#pragma unroll
            for (int e = 0; e < N; ++e) part[0][e] = v[e];
        } else {
            typedef T Pair __attribute__((ext_vector_type(2)));
            unsigned word[PARTS][N / 2];
#pragma unroll
            for (int e = 0; e < N; e += 2) {
                float x = v[e], y = v[e + 1];
                // (a product behind them has to be rounded to fp32 here: folded into the conversion to fp16 it rounds once, where the
                // difference below sees it rounded twice, and one value in some thousands lost its second part)
                if constexpr (kNormalise) asm("" : "+v"(x), "+v"(y));
#pragma unroll
                for (int p = 0; p < PARTS; ++p) {
                    const Pair r = {Tr::from_f32(x), Tr::from_f32(y)};
                    unsigned w = __builtin_bit_cast(unsigned, r);
                    if (p + 1 < PARTS) {
                        asm("" : "+v"(w));
                        if constexpr (kNormalise) {
                            const Pair back = __builtin_bit_cast(Pair, w);
                            x -= (float)back[0];
                            y -= (float)back[1];
                        } else {
                            x -= __builtin_bit_cast(float, w << 16);
                            y -= __builtin_bit_cast(float, w & 0xffff0000u);
                        }
                    }
                    word[p][e / 2] = w;
                }
            }
#pragma unroll
            for (int p = 0; p < PARTS; ++p) __builtin_memcpy(&part[p], word[p], sizeof(V));
        }
    }
};

// A chunk's running gates, in LDS: exponents (base 2) from the chunk's start to each row, as a float and what it leaves out of the
// double that they are summed in, so that differences stay exact behind a gate that forgets everything.
//
// The state is kept as 2^base times what stands in registers: while base stays small, a chunk's gates move base instead of multiplying every
// element, and the rows' weights make up for it.  |base| < 16 leaves fp32's range to the state but for that factor, and mild gates reach it
// once in several chunks.
struct Gates {
    float hi[kChunk], lo[kChunk];
    float in[kChunk];               // the state's factor in this row's output
    float weight[kChunk];           // this row's factor in the state behind the chunk
    float total, grow, exponent, unit;      // what the registers are multiplied by; how far gates above 0 let a weight grow; log2 of the chunk's
                                            // gates; 2^base behind the chunk
};
constexpr float kMostBase = 16.0f;

constexpr double kLog2e = 1.4426950408889634;

// v of the lane that a data-parallel move takes it from; 0 where it takes none
template <int CTRL, int ROWS>
__device__ __forceinline__ float moved(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, false));
}
template <int CTRL, int ROWS>
__device__ __forceinline__ double moved(double v) {
    const unsigned long long u = __builtin_bit_cast(unsigned long long, v);
    const unsigned lo = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)u, CTRL, ROWS, 0xf, false);
    const unsigned hi = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)(u >> 32), CTRL, ROWS, 0xf, false);
    return __builtin_bit_cast(double, (unsigned long long)hi << 32 | lo);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ unsigned moved(unsigned v) {
    return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false);
}
// sum over this lane and those before it
template <class V>
__device__ __forceinline__ V running_sum(V v) {
    v += moved<0x111, 0xf>(v);      // row_shr 1, 2, 4, 8: within 16 lanes
    v += moved<0x112, 0xf>(v);
    v += moved<0x114, 0xf>(v);
    v += moved<0x118, 0xf>(v);
    v += moved<0x142, 0xa>(v);      // row_bcast 15: the last lane of rows 0 and 2 to rows 1 and 3
    v += moved<0x143, 0xc>(v);      // row_bcast 31: that of row 1 to rows 2 and 3
    return v;
}

// the largest of this lane and those before it
__device__ __forceinline__ unsigned running_max(unsigned v) {
    v = max(v, moved<0x111, 0xf>(v));
    v = max(v, moved<0x112, 0xf>(v));
    v = max(v, moved<0x114, 0xf>(v));
    v = max(v, moved<0x118, 0xf>(v));
    v = max(v, moved<0x142, 0xa>(v));
    v = max(v, moved<0x143, 0xc>(v));
    return v;
}

// By one wave; `g`: this lane's row's gate (0 where there is no row); base: before the chunk, and then behind it.  LAZY: base may move.
template <bool LAZY>
__device__ __forceinline__ void run_gates(Gates* out, float g, int reverse, float in_scale, float weight_scale, bool want_grow, double& base) {
    const int lane = lane_id_again();
    double own = (double)g * kLog2e;
    if (own < -150.0) own = -150.0;         // 2^-150 is 0 in fp32; a NaN stays one
    const double sum = running_sum(own);
    const unsigned long long last = __builtin_bit_cast(unsigned long long, sum);
    const double total = __builtin_bit_cast(double, (unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)(unsigned)(last >> 32), 63) << 32 |
                                                        (unsigned)__builtin_amdgcn_readlane((int)(unsigned)last, 63));
    const double here = reverse ? sum - own : sum;
    const float hi = (float)here, lo = (float)(here - (double)hi);
    out->hi[lane] = hi;
    out->lo[lane] = lo;
    const double in = here + base;
    const float in_hi = (float)in;
    out->in[lane] = __builtin_amdgcn_exp2f(in_hi) * fmaf((float)(in - (double)in_hi), 0.693147182f, 1.0f) * in_scale;
    const double moved = base + total;
    const bool moves = LAZY && moved > -kMostBase && moved < kMostBase;
    const double weight = moves ? -in : total - here;
    const float w_hi = (float)weight;
    out->weight[lane] = __builtin_amdgcn_exp2f(w_hi) * fmaf((float)(weight - (double)w_hi), 0.693147182f, 1.0f) * weight_scale;
    base = moves ? moved : 0.0;
    if (lane == 0) {
        out->total = moves ? 1.0f : __builtin_amdgcn_exp2f((float)moved);
        out->exponent = (float)total;
        out->unit = __builtin_amdgcn_exp2f((float)base);
    }
    if (want_grow) {
        const float grow = running_sum(own > 0.0 ? (float)own : 0.0f);
        if (lane == 63) out->grow = __builtin_amdgcn_exp2f(grow);
    }
}

// a power of two that takes values up to `bound` to at most 2^top (by default fp16's range); 1 where there is no such bound
__device__ __forceinline__ float normaliser(float bound, int top = 15) {
    if (!(bound > 0.0f) || !(bound < 3e38f)) return 1.0f;
    int e = (int)(__builtin_bit_cast(unsigned, bound) >> 23) - 126;      // bound < 2^e
    e = top - e;
    e = e < -120 ? -120 : (e > 100 ? 100 : e);
    return __builtin_bit_cast(float, (unsigned)(e + 127) << 23);
}
// What a state of fp16 inputs is multiplied by while it stands in registers: as much as takes what is added next (up to `bound`) to fp16's range,
// but no more than leaves the state (up to `state`) in fp32's.  `before`: what it is now.
__device__ __forceinline__ float unit_of(float bound, float state, float before) {
    const float u = bound > 0.0f ? normaliser(bound) : before;
    return state * u > 0x1p100f && state < 3e38f ? normaliser(state, 100) : u;
}

__device__ __forceinline__ float half_bits(unsigned b) { return (float)__builtin_bit_cast(_Float16, (unsigned short)b); }

}  // namespace rec
}  // namespace msla
