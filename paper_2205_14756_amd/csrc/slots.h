// How sequences packed behind each other are dealt to workgroups: in runs ("slots") of `run` tokens of one sequence.  Sequence b has the slots from
// first_slot(b) on, as many as it needs; those between its last one and first_slot(b + 1) have no tokens.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace msla {

struct Slots {
    const int* offsets;         // or NULL: equal lengths
    int sequences, tokens, run;
    int each;                   // slots of a sequence (equal lengths)
};

// (host) the slots of `s`, at most
inline int64_t slot_count(const Slots& s) {
    return s.offsets ? (int64_t)s.tokens / s.run + s.sequences : (int64_t)s.sequences * s.each;
}
inline Slots slots_of(const int* offsets, int sequences, int64_t tokens, int run) {
    const int64_t length = tokens / sequences;
    return Slots{offsets, sequences, (int)tokens, run, (int)(length <= run ? 1 : (length + run - 1) / run)};
}

__device__ __forceinline__ int clamp_to(int v, int lo, int hi) { return v < lo ? lo : (v > hi ? hi : v); }
// rows of sequence b, within the buffers whatever the array holds
__device__ __forceinline__ void rows_of_sequence(const Slots& s, int b, int& lo, int& hi) {
    if (s.offsets) {
        lo = clamp_to(s.offsets[b], 0, s.tokens);
        hi = clamp_to(s.offsets[b + 1], lo, s.tokens);
    } else {
        const int length = s.tokens / s.sequences;
        lo = b * length;
        hi = lo + length;
    }
}
__device__ __forceinline__ int first_slot(const Slots& s, int b) {
    return s.offsets ? clamp_to(s.offsets[b], 0, s.tokens) / s.run + b : b * s.each;
}

// A slot's sequence (its rows lo to hi) and tokens (from to until; none in a slot that is not used, whose `used` is false: an empty sequence
// has one that is).
struct Slot {
    int sequence, index, lo, hi, from, until;
    bool used, first, last;
};
__device__ __forceinline__ Slot slot_at(const Slots& s, int slot) {
    Slot o;
    int b;
    if (s.offsets) {
        int top = s.sequences;              // the last sequence whose first slot is not behind this one
        b = 0;
        while (top - b > 1) {
            const int mid = b + (top - b) / 2;
            if (first_slot(s, mid) <= slot) b = mid;
            else top = mid;
        }
    } else {
        b = slot / s.each;
    }
    rows_of_sequence(s, b, o.lo, o.hi);
    o.sequence = b;
    o.index = slot - first_slot(s, b);
    const int64_t from = (int64_t)o.lo + (int64_t)o.index * s.run;
    o.used = o.index == 0 || (o.index > 0 && from < o.hi);
    o.from = o.used ? (int)from : o.hi;
    o.until = o.hi - o.from < s.run ? o.hi : o.from + s.run;
    o.first = o.index == 0;
    o.last = o.used && o.until == o.hi;
    return o;
}

}  // namespace msla
