// Host side of the part of include/msla_sequence.h that a selective state space layer is made of: argument validation, how scans and convolutions are
// cut into slots, workspace carving.  Like msla_sequence.cpp: no allocation, no synchronisation, no state that depends on a call's arguments, and every
// failure before the first launch leaves the stream untouched.
#include "../../include/msla_sequence.h"

#include <math.h>

#include "msla_layer_kernels.h"
#include "msla_sequence_kernels.h"

namespace {

using msla::ConvCall;
using msla::LayerNormCall;
using msla::ScanCall;
using msla::Slots;
using msla::TokenRows;

constexpr size_t kAlign = 256;
constexpr int64_t kMost = (int64_t)1 << 46;             // elements that a buffer may span
constexpr int64_t kMostTokens = 0x7fffffffLL - 4096;    // (token numbers, and those of some tokens behind the last, are ints)
constexpr int kMostChannels = 1 << 20;
constexpr int64_t kMostGroups = (int64_t)1 << 23;       // workgroups of a launch: fewer than 2^32 threads, at most 512 to a group
constexpr int64_t kUnits = 256;                         // compute units of an MI355X
constexpr int64_t kCutTokens = 96;                      // what a scan's two more launches take, in tokens of one slot

size_t align_up(size_t v) { return (v + kAlign - 1) / kAlign * kAlign; }
bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
bool known(msla_dtype dt) { return dt == MSLA_F32 || dt == MSLA_F16 || dt == MSLA_BF16; }
size_t elem_size(msla_dtype dt) { return dt == MSLA_F32 ? 4 : 2; }
msla_status status_of(hipError_t e) { return e == hipSuccess ? MSLA_OK : MSLA_ERR_LAUNCH; }
TokenRows rows_of(const msla_rows& r) { return TokenRows{r.data, r.token_stride}; }
bool same(const msla_rows& a, const msla_rows& b) { return a.data != nullptr && a.data == b.data; }

msla_status check_sequences(int sequences, int64_t tokens, const int32_t* offsets) {
    if (sequences <= 0 || tokens < 0 || !aligned(offsets, 4)) return MSLA_ERR_INVALID_ARG;
    if (offsets == nullptr && tokens % sequences != 0) return MSLA_ERR_INVALID_ARG;
    return tokens > kMostTokens ? MSLA_ERR_UNSUPPORTED : MSLA_OK;
}

// further apart than a lane's 32-bit offset reaches over a scan's tile of 64 tokens
bool wide(const msla_rows& r, int64_t tokens, msla_dtype dt) { return tokens > 1 && r.token_stride * (int64_t)elem_size(dt) >= (int64_t)1 << 24; }

// rows of `width` elements; where they are written they lie apart
bool fits(const msla_rows& r, int64_t tokens, int64_t width, msla_dtype dt, bool written) {
    if (tokens == 0) return true;
    if (r.data == nullptr || !aligned(r.data, elem_size(dt)) || r.token_stride < 0 || r.token_stride > kMost / tokens) return false;
    return !written || tokens == 1 || r.token_stride >= width;
}

msla_status check_scan(const msla_selective_scan* s, msla_dtype dt) {
    if (s == nullptr || !known(dt)) return MSLA_ERR_INVALID_ARG;
    if (s->channels <= 0 || s->groups <= 0 || s->states <= 0 || s->channels % s->groups != 0 || (s->softplus != 0 && s->softplus != 1))
        return MSLA_ERR_INVALID_ARG;
    const msla_status st = check_sequences(s->sequences, s->tokens, s->offsets);
    if (st != MSLA_OK) return st;
    if (s->states != 8 && s->states != 16 && s->states != 32 && s->states != 64) return MSLA_ERR_UNSUPPORTED;
    if (s->channels > kMostChannels) return MSLA_ERR_UNSUPPORTED;
    return MSLA_OK;
}

struct ScanPlan {
    Slots slots;
    bool cut;
    int64_t count;                  // slots
    Slots marks;
    size_t states_at, d_states_at, steps_at, marks_at, mark_steps_at, parts_at, shared_at, bytes;
};

// How long slots are.  Two workgroups fill a compute unit (one of fp32 with 64 states and one of the gradient's pass back, whose registers leave no more: the
// same plan serves them, a unit's two in turn).  A sequence that is cut does 1.65 times its work, in the gradient 1.2 times, and two (one) more
// launches.  Equal sequences are cut into as many slots as leave every unit two workgroups at most, if that is worth it; packed ones, whose lengths nobody
// knows here, into runs of a share of what a unit has to do (those that are no longer run whole).  us with a whole share, half of one, a quarter: 24 sequences of
// 5003 tokens, 2048 channels of 64 states 211 / 245 / 267, 16 of 8192 tokens, 4096 channels 225 / 281 / 275; but of fewer sequences than fill the units, 8 of 4096,
// 1024 channels 78 / 59 / 59, 2 of 8000, 2048 channels 189 / 152 / 153; the gradient of the second one 999 / 982 / 941, of the third 181 / 155 / 149.
msla_status plan_of(const msla_selective_scan& s, bool backward, ScanPlan* p) {
    const int64_t tiles = msla::scan_tiles(s.channels, s.groups), tile = 4 * msla::scan_lanes(s.states);      // (tokens of a tile)
    const int64_t longest = s.offsets ? s.tokens : s.tokens / s.sequences, each = 2 * kUnits / (s.sequences * tiles);
    auto whole_tiles = [&](int64_t tokens) { return (tokens + tile - 1) / tile * tile; };
    const int64_t shares = backward ? 4 : (s.sequences * tiles >= 2 * kUnits ? 1 : 2);
    int64_t run = s.offsets ? whole_tiles(s.tokens * tiles / (shares * kUnits) + 1) : whole_tiles(longest / (each > 0 ? each : 1) + 1);
    p->cut = s.offsets ? longest > run : each >= 2 && longest * 100 > run * (backward ? 120 : 165) + kCutTokens * 100;
    if (!p->cut) run = whole_tiles(longest + 1);
    p->slots = msla::slots_of(s.offsets, s.sequences, s.tokens, (int)run);
    p->count = msla::slot_count(p->slots);
    const int64_t per_state = (int64_t)s.channels * s.states;
    if (p->count * tiles >= kMostGroups || (int64_t)s.sequences * ((per_state + 255) / 256) >= kMostGroups) return MSLA_ERR_UNSUPPORTED;
    if (backward && (s.tokens * (int64_t)s.groups * s.states * 2 + 255) / 256 >= kMostGroups) return MSLA_ERR_UNSUPPORTED;
    size_t at = 0;
    auto take = [&](size_t floats) {
        const size_t here = at;
        at += align_up(floats * 4);
        return here;
    };
    p->states_at = p->d_states_at = p->steps_at = p->marks_at = p->mark_steps_at = p->parts_at = p->shared_at = 0;
    if (p->cut) {
        p->states_at = take((size_t)p->count * per_state);
        if (backward) p->d_states_at = take((size_t)p->count * per_state);
        p->steps_at = take((size_t)p->count * s.channels);
    }
    if (backward) {
        p->marks = msla::slots_of(s.offsets, s.sequences, s.tokens, msla::scan_lanes(s.states));
        const size_t marks = (size_t)msla::slot_count(p->marks);
        p->marks_at = take(marks * per_state);
        if (p->cut) p->mark_steps_at = take(marks * s.channels);
        p->parts_at = take((size_t)p->count * (per_state + 2 * s.channels));
        p->shared_at = take((size_t)tiles * s.tokens * 2 * s.states);
    }
    p->bytes = at;
    return MSLA_OK;
}

ScanCall call_of(const msla_selective_scan& s, msla_rows x, msla_rows delta, const float* a, msla_rows b, msla_rows c, const float* skip,
                 const float* delta_bias, msla_rows gate, const float* initial) {
    ScanCall k = {};
    k.channels = s.channels;
    k.groups = s.groups;
    k.states = s.states;
    k.softplus = s.softplus;
    k.x = rows_of(x);
    k.delta = rows_of(delta);
    k.b = rows_of(b);
    k.c = rows_of(c);
    k.gate = rows_of(gate);
    k.a = a;
    k.skip = skip;
    k.bias = delta_bias;
    k.initial = initial;
    return k;
}

bool inputs_fit(const msla_selective_scan& s, const msla_rows& x, const msla_rows& delta, const float* a, const msla_rows& b, const msla_rows& c,
                const float* skip, const float* delta_bias, const msla_rows& gate, const float* initial, msla_dtype dt) {
    const int64_t shared = (int64_t)s.groups * s.states;
    if (a == nullptr || !aligned(a, 4) || !aligned(skip, 4) || !aligned(delta_bias, 4) || !aligned(initial, 4)) return false;
    if (gate.data != nullptr && !fits(gate, s.tokens, s.channels, dt, false)) return false;
    return fits(x, s.tokens, s.channels, dt, false) && fits(delta, s.tokens, s.channels, dt, false) && fits(b, s.tokens, shared, dt, false) &&
           fits(c, s.tokens, shared, dt, false);
}

void place(ScanCall* k, const ScanPlan& p, void* workspace) {
    char* ws = (char*)workspace;
    k->slots = p.slots;
    k->cut = p.cut;
    k->states_at = (float*)(ws + p.states_at);
    k->d_states_at = (float*)(ws + p.d_states_at);
    k->steps_at = (float*)(ws + p.steps_at);
    k->marks = p.marks;
    k->marks_at = (float*)(ws + p.marks_at);
    k->mark_steps_at = (float*)(ws + p.mark_steps_at);
    k->parts_at = (float*)(ws + p.parts_at);
    k->shared_at = (float*)(ws + p.shared_at);
}

msla_status check_conv(const msla_causal_conv* s, msla_dtype dt) {
    if (s == nullptr || !known(dt) || s->channels <= 0 || s->width <= 0 || (s->silu != 0 && s->silu != 1)) return MSLA_ERR_INVALID_ARG;
    const msla_status st = check_sequences(s->sequences, s->tokens, s->offsets);
    if (st != MSLA_OK) return st;
    if (s->width < 2 || s->width > 4 || s->channels > kMostChannels) return MSLA_ERR_UNSUPPORTED;
    return MSLA_OK;
}

// Runs of tokens: the longest ones (each reads width - 1 rows again) that leave `want` waves.
int conv_run(const msla_causal_conv& s, msla_dtype dt, int most, int64_t want) {
    const int64_t pieces = (s.channels * (int64_t)elem_size(dt) + 15) / 16;
    int run = most;
    while (run > 4 && s.tokens / run * pieces < 64 * want) run /= 2;
    return run;
}
constexpr int kConvRun = 32, kConvRunBackward = 64;
constexpr int64_t kConvWaves = 2048;

msla_status conv_slots(const msla_causal_conv& s, msla_dtype dt, bool backward, Slots* slots) {
    *slots = msla::slots_of(s.offsets, s.sequences, s.tokens, conv_run(s, dt, backward ? kConvRunBackward : kConvRun, kConvWaves));
    // (a workgroup has 256 pieces of 16 or 8 bytes, or less where a row is no power of two of them)
    return msla::slot_count(*slots) * (((int64_t)s.channels * (int64_t)elem_size(dt) + 7) / 8 * 2 + 256) / 256 >= kMostGroups ? MSLA_ERR_UNSUPPORTED : MSLA_OK;
}

ConvCall call_of(const msla_causal_conv& s, msla_rows x, const void* weight, const void* bias, const void* initial) {
    ConvCall k = {};
    k.channels = s.channels;
    k.width = s.width;
    k.silu = s.silu;
    k.x = rows_of(x);
    k.weight = weight;
    k.bias = bias;
    k.initial = initial;
    return k;
}

msla_status check_rows(int64_t rows, int channels, float eps, msla_dtype dt) {
    if (rows < 0 || channels <= 0 || !(eps >= 0.0f) || !(eps < INFINITY) || !known(dt)) return MSLA_ERR_INVALID_ARG;
    if (channels > 32768 || rows > 0x7fffffffLL) return MSLA_ERR_UNSUPPORTED;
    return MSLA_OK;
}

}  // namespace

extern "C" {

msla_status msla_selective_scan_workspace_bytes(const msla_selective_scan* shape, int backward, msla_dtype dt, size_t* bytes) {
    if (bytes == nullptr) return MSLA_ERR_INVALID_ARG;
    msla_status st = check_scan(shape, dt);
    if (st != MSLA_OK) return st;
    ScanPlan plan;
    st = plan_of(*shape, backward != 0, &plan);
    if (st == MSLA_OK) *bytes = plan.bytes;
    return st;
}

msla_status msla_selective_scan_forward(const msla_selective_scan* shape, msla_rows x, msla_rows delta, const float* a, msla_rows b, msla_rows c,
                                        const float* skip, const float* delta_bias, msla_rows gate, const float* initial_state, msla_rows out,
                                        float* final_state, void* workspace, size_t workspace_bytes, msla_dtype dt, void* stream) {
    msla_status st = check_scan(shape, dt);
    if (st != MSLA_OK) return st;
    const msla_selective_scan& s = *shape;
    if (!inputs_fit(s, x, delta, a, b, c, skip, delta_bias, gate, initial_state, dt) || !fits(out, s.tokens, s.channels, dt, true) ||
        !aligned(final_state, 4) || same(out, b) || same(out, c))
        return MSLA_ERR_INVALID_ARG;
    for (const msla_rows* i : {&x, &delta, &gate})
        if (same(out, *i)) return MSLA_ERR_INVALID_ARG;
    for (const msla_rows* r : {&x, &delta, &gate, &out})
        if (wide(*r, s.tokens, dt)) return MSLA_ERR_UNSUPPORTED;
    ScanPlan plan;
    st = plan_of(s, false, &plan);
    if (st != MSLA_OK) return st;
    if (plan.bytes > 0 && (workspace == nullptr || !aligned(workspace, 16))) return MSLA_ERR_INVALID_ARG;
    if (workspace_bytes < plan.bytes) return MSLA_ERR_WORKSPACE;
    ScanCall k = call_of(s, x, delta, a, b, c, skip, delta_bias, gate, initial_state);
    place(&k, plan, workspace);
    k.out = rows_of(out);
    k.final_state = final_state;
    return status_of(msla::launch_scan_forward((int)dt, k, (hipStream_t)stream));
}

msla_status msla_selective_scan_backward(const msla_selective_scan* shape, msla_rows x, msla_rows delta, const float* a, msla_rows b, msla_rows c,
                                         const float* skip, const float* delta_bias, msla_rows gate, const float* initial_state, msla_rows d_out,
                                         const float* d_final_state, msla_rows d_x, msla_rows d_delta, float* d_a, msla_rows d_b, msla_rows d_c,
                                         float* d_skip, float* d_delta_bias, msla_rows d_gate, float* d_initial_state, void* workspace,
                                         size_t workspace_bytes, msla_dtype dt, void* stream) {
    msla_status st = check_scan(shape, dt);
    if (st != MSLA_OK) return st;
    const msla_selective_scan& s = *shape;
    const int64_t shared = (int64_t)s.groups * s.states;
    if (!inputs_fit(s, x, delta, a, b, c, skip, delta_bias, gate, initial_state, dt) || !fits(d_out, s.tokens, s.channels, dt, false) ||
        !fits(d_x, s.tokens, s.channels, dt, true) || !fits(d_delta, s.tokens, s.channels, dt, true) || !fits(d_b, s.tokens, shared, dt, true) ||
        !fits(d_c, s.tokens, shared, dt, true) || !aligned(d_a, 4) || !aligned(d_skip, 4) || !aligned(d_delta_bias, 4) ||
        !aligned(d_final_state, 4) || !aligned(d_initial_state, 4))
        return MSLA_ERR_INVALID_ARG;
    if ((gate.data != nullptr) != (d_gate.data != nullptr) && s.tokens > 0) return MSLA_ERR_INVALID_ARG;
    if (gate.data != nullptr && !fits(d_gate, s.tokens, s.channels, dt, true)) return MSLA_ERR_INVALID_ARG;
    if (d_initial_state != nullptr && (d_initial_state == d_final_state || d_initial_state == initial_state)) return MSLA_ERR_INVALID_ARG;
    const msla_rows* const outs[] = {&d_x, &d_delta, &d_b, &d_c, &d_gate};
    for (int o = 0; o < 5; ++o) {
        for (const msla_rows* i : {&x, &delta, &b, &c, &gate, &d_out})
            if (same(*outs[o], *i)) return MSLA_ERR_INVALID_ARG;
        for (int other = 0; other < o; ++other)
            if (same(*outs[o], *outs[other])) return MSLA_ERR_INVALID_ARG;
    }
    for (const msla_rows* r : {&x, &delta, &gate, &d_out, &d_x, &d_delta, &d_gate})
        if (wide(*r, s.tokens, dt)) return MSLA_ERR_UNSUPPORTED;
    ScanPlan plan;
    st = plan_of(s, true, &plan);
    if (st != MSLA_OK) return st;
    if (workspace == nullptr || !aligned(workspace, 16)) return MSLA_ERR_INVALID_ARG;
    if (workspace_bytes < plan.bytes) return MSLA_ERR_WORKSPACE;
    ScanCall k = call_of(s, x, delta, a, b, c, skip, delta_bias, gate, initial_state);
    place(&k, plan, workspace);
    k.d_out = rows_of(d_out);
    k.d_final = d_final_state;
    k.d_x = rows_of(d_x);
    k.d_delta = rows_of(d_delta);
    k.d_b = rows_of(d_b);
    k.d_c = rows_of(d_c);
    k.d_gate = rows_of(d_gate);
    k.d_a = d_a;
    k.d_skip = d_skip;
    k.d_bias = d_delta_bias;
    k.d_initial = d_initial_state;
    return status_of(msla::launch_scan_backward((int)dt, k, (hipStream_t)stream));
}

msla_status msla_selective_scan_step(const msla_selective_scan* shape, msla_rows x, msla_rows delta, const float* a, msla_rows b, msla_rows c,
                                     const float* skip, const float* delta_bias, msla_rows gate, const float* state, msla_rows out, float* new_state,
                                     msla_dtype dt, void* stream) {
    const msla_status st = check_scan(shape, dt);
    if (st != MSLA_OK) return st;
    const msla_selective_scan& s = *shape;
    if (s.offsets != nullptr || s.tokens != s.sequences || state == nullptr || new_state == nullptr || !aligned(new_state, 4))
        return MSLA_ERR_INVALID_ARG;
    if (!inputs_fit(s, x, delta, a, b, c, skip, delta_bias, gate, state, dt) || !fits(out, s.tokens, s.channels, dt, true) || same(out, b) || same(out, c))
        return MSLA_ERR_INVALID_ARG;
    for (const msla_rows* i : {&x, &delta, &gate})
        if (same(out, *i)) return MSLA_ERR_INVALID_ARG;
    if ((int64_t)s.sequences * ((s.channels + 63) / 64) >= kMostGroups) return MSLA_ERR_UNSUPPORTED;
    ScanCall k = call_of(s, x, delta, a, b, c, skip, delta_bias, gate, state);
    k.slots = msla::slots_of(nullptr, s.sequences, s.tokens, 1);
    k.out = rows_of(out);
    k.final_state = new_state;
    return status_of(msla::launch_scan_step((int)dt, k, (hipStream_t)stream));
}

msla_status msla_causal_conv_forward(const msla_causal_conv* shape, msla_rows x, const void* weight, const void* bias, const void* initial_state,
                                     msla_rows out, void* final_state, msla_dtype dt, void* stream) {
    msla_status st = check_conv(shape, dt);
    if (st != MSLA_OK) return st;
    const msla_causal_conv& s = *shape;
    const size_t e = elem_size(dt);
    if (weight == nullptr || !aligned(weight, e) || !aligned(bias, e) || !aligned(initial_state, e) || !aligned(final_state, e) ||
        !fits(x, s.tokens, s.channels, dt, false) || !fits(out, s.tokens, s.channels, dt, true) || same(out, x) ||
        (final_state != nullptr && final_state == initial_state))
        return MSLA_ERR_INVALID_ARG;
    ConvCall k = call_of(s, x, weight, bias, initial_state);
    st = conv_slots(s, dt, false, &k.slots);
    if (st != MSLA_OK) return st;
    k.out = rows_of(out);
    k.final_state = final_state;
    return status_of(msla::launch_conv_forward((int)dt, k, (hipStream_t)stream));
}

msla_status msla_causal_conv_backward_workspace_bytes(const msla_causal_conv* shape, msla_dtype dt, size_t* bytes) {
    if (bytes == nullptr) return MSLA_ERR_INVALID_ARG;
    msla_status st = check_conv(shape, dt);
    if (st != MSLA_OK) return st;
    Slots slots;
    st = conv_slots(*shape, dt, true, &slots);
    if (st == MSLA_OK) *bytes = align_up((size_t)msla::slot_count(slots) * shape->channels * (shape->width + 1) * 4);
    return st;
}

msla_status msla_causal_conv_backward(const msla_causal_conv* shape, msla_rows x, const void* weight, const void* bias, const void* initial_state,
                                      msla_rows d_out, const void* d_final_state, msla_rows d_x, float* d_weight, float* d_bias,
                                      void* d_initial_state, void* workspace, size_t workspace_bytes, msla_dtype dt, void* stream) {
    msla_status st = check_conv(shape, dt);
    if (st != MSLA_OK) return st;
    const msla_causal_conv& s = *shape;
    const size_t e = elem_size(dt);
    if (weight == nullptr || !aligned(weight, e) || !aligned(bias, e) || !aligned(initial_state, e) || !aligned(d_final_state, e) ||
        !aligned(d_initial_state, e) || !aligned(d_weight, 4) || !aligned(d_bias, 4) || !fits(x, s.tokens, s.channels, dt, false) ||
        !fits(d_out, s.tokens, s.channels, dt, false) || !fits(d_x, s.tokens, s.channels, dt, true) || same(d_x, x) || same(d_x, d_out))
        return MSLA_ERR_INVALID_ARG;
    if (d_initial_state != nullptr && (d_initial_state == d_final_state || d_initial_state == initial_state)) return MSLA_ERR_INVALID_ARG;
    ConvCall k = call_of(s, x, weight, bias, initial_state);
    st = conv_slots(s, dt, true, &k.slots);
    if (st != MSLA_OK) return st;
    if (d_weight != nullptr || d_bias != nullptr) {
        if (workspace == nullptr || !aligned(workspace, 16)) return MSLA_ERR_INVALID_ARG;
        if (workspace_bytes < (size_t)msla::slot_count(k.slots) * s.channels * (s.width + 1) * 4) return MSLA_ERR_WORKSPACE;
        k.parts_at = (float*)workspace;
    }
    k.d_out = rows_of(d_out);
    k.d_x = rows_of(d_x);
    k.d_final = d_final_state;
    k.d_initial = d_initial_state;
    k.d_weight = d_weight;
    k.d_bias = d_bias;
    return status_of(msla::launch_conv_backward((int)dt, k, (hipStream_t)stream));
}

msla_status msla_causal_conv_step(const msla_causal_conv* shape, msla_rows x, const void* weight, const void* bias, const void* state, msla_rows out,
                                  void* new_state, msla_dtype dt, void* stream) {
    msla_status st = check_conv(shape, dt);
    if (st != MSLA_OK) return st;
    const msla_causal_conv& s = *shape;
    const size_t e = elem_size(dt);
    if (s.offsets != nullptr || s.tokens != s.sequences || weight == nullptr || state == nullptr || new_state == nullptr || !aligned(weight, e) ||
        !aligned(bias, e) || !aligned(state, e) || !aligned(new_state, e) || !fits(x, s.tokens, s.channels, dt, false) ||
        !fits(out, s.tokens, s.channels, dt, true) || same(out, x))
        return MSLA_ERR_INVALID_ARG;
    ConvCall k = call_of(s, x, weight, bias, state);
    st = conv_slots(s, dt, false, &k.slots);
    if (st != MSLA_OK) return st;
    k.out = rows_of(out);
    k.final_state = new_state;
    return status_of(msla::launch_conv_step((int)dt, k, (hipStream_t)stream));
}

msla_status msla_layer_norm_forward(const void* x, const void* residual, const void* weight, const void* bias, void* y, void* sum, int64_t rows,
                                    int channels, float eps, msla_dtype dt, void* stream) {
    const msla_status st = check_rows(rows, channels, eps, dt);
    if (st != MSLA_OK) return st;
    const size_t e = elem_size(dt);
    for (const void* p : {x, residual, weight, bias, (const void*)y, (const void*)sum})
        if (!aligned(p, e)) return MSLA_ERR_INVALID_ARG;
    if (rows == 0) return MSLA_OK;
    if (x == nullptr || y == nullptr || y == sum || (residual != nullptr && y == residual)) return MSLA_ERR_INVALID_ARG;
    const LayerNormCall c = {x, residual, weight, bias, y, sum, rows, channels, eps};
    return status_of(msla::launch_layer_norm((int)dt, c, (hipStream_t)stream));
}

msla_status msla_layer_norm_backward_workspace_bytes(int64_t rows, int channels, msla_dtype dt, size_t* bytes) {
    if (bytes == nullptr) return MSLA_ERR_INVALID_ARG;
    const msla_status st = check_rows(rows, channels, 0.0f, dt);
    if (st == MSLA_OK) *bytes = align_up((size_t)msla::layer_norm_blocks(rows, channels, (int)elem_size(dt)) * channels * 8);
    return st;
}

msla_status msla_layer_norm_backward(const void* sum, const void* weight, const void* d_y, const void* d_sum, void* d_r, float* d_weight, float* d_bias,
                                     void* workspace, size_t workspace_bytes, int64_t rows, int channels, float eps, msla_dtype dt, void* stream) {
    const msla_status st = check_rows(rows, channels, eps, dt);
    if (st != MSLA_OK) return st;
    const size_t e = elem_size(dt);
    for (const void* p : {sum, weight, d_y, d_sum, (const void*)d_r})
        if (!aligned(p, e)) return MSLA_ERR_INVALID_ARG;
    if (!aligned(d_weight, 4) || !aligned(d_bias, 4)) return MSLA_ERR_INVALID_ARG;
    if (rows > 0 && (sum == nullptr || d_y == nullptr || d_r == nullptr || d_r == sum)) return MSLA_ERR_INVALID_ARG;
    if ((d_weight != nullptr || d_bias != nullptr) && rows > 0) {
        if (workspace == nullptr || !aligned(workspace, 16)) return MSLA_ERR_INVALID_ARG;
        if (workspace_bytes < (size_t)msla::layer_norm_blocks(rows, channels, (int)e) * channels * 8) return MSLA_ERR_WORKSPACE;
    }
    return status_of(msla::launch_layer_norm_backward((int)dt, sum, weight, d_y, d_sum, d_r, d_weight, d_bias, (float*)workspace, rows, channels, eps,
                                                      (hipStream_t)stream));
}

msla_status msla_quantize_rows_integer(const void* x, void* x8, float* scale, int64_t rows, int channels, msla_dtype dt, void* stream) {
    const msla_status st = check_rows(rows, channels, 0.0f, dt);
    if (st != MSLA_OK) return st;
    if (!aligned(x, elem_size(dt)) || !aligned(scale, 4)) return MSLA_ERR_INVALID_ARG;
    if (rows == 0) return MSLA_OK;
    if (x == nullptr || x8 == nullptr || scale == nullptr || x8 == x) return MSLA_ERR_INVALID_ARG;
    return status_of(msla::launch_quantize_integer((int)dt, x, x8, scale, rows, channels, (hipStream_t)stream));
}

msla_status msla_linear_integer(const void* x8, const float* x_scale, const void* w8, const float* w_scale, void* y, int64_t rows, int c_in, int c_out,
                                msla_dtype dt, void* stream) {
    if (rows < 0 || c_in <= 0 || c_out <= 0 || !known(dt)) return MSLA_ERR_INVALID_ARG;
    if (!aligned(x8, 16) || !aligned(w8, 16) || !aligned(y, 16) || !aligned(x_scale, 4) || !aligned(w_scale, 4)) return MSLA_ERR_INVALID_ARG;
    // (128 * 128 * 131072 is 2^31)
    if (c_in % 16 != 0 || c_out % 16 != 0 || c_in >= 131072 || c_out > kMostChannels || rows > 0x7fffffffLL) return MSLA_ERR_UNSUPPORTED;
    if (rows == 0) return MSLA_OK;
    if (!x8 || !x_scale || !w8 || !w_scale || !y || y == x8 || y == w8) return MSLA_ERR_INVALID_ARG;
    return status_of(msla::launch_linear_integer((int)dt, x8, x_scale, w8, w_scale, y, rows, c_in, c_out, (hipStream_t)stream));
}

}  // extern "C"
