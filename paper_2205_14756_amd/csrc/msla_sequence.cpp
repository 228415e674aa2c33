// Host side of the C ABI declared in include/msla_sequence.h: argument validation, how a scan is cut into segments, workspace
// carving.  Like msla_api.cpp: no allocation, no synchronisation, no state that depends on a call's arguments, and every failure before
// the first launch leaves the stream untouched.
#include "../../include/msla_sequence.h"

#include <math.h>

#include "msla_sequence_kernels.h"

namespace {

using msla::NormCall;
using msla::RecurrenceCall;
using msla::RecurrencePlan;
using msla::RecurrenceRows;

constexpr size_t kAlign = 256;
constexpr int64_t kMost = (int64_t)1 << 46;         // elements that a buffer may span

size_t align_up(size_t v) { return (v + kAlign - 1) / kAlign * kAlign; }
bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
bool known(msla_dtype dt) { return dt == MSLA_F32 || dt == MSLA_F16 || dt == MSLA_BF16; }
size_t elem_size(msla_dtype dt) { return dt == MSLA_F32 ? 4 : 2; }
msla_status status_of(hipError_t e) { return e == hipSuccess ? MSLA_OK : MSLA_ERR_LAUNCH; }

// Workgroups that a scan should have at least: two for each of an MI355X's 256 compute units.
constexpr int64_t kWantGroups = 512;
// Steps of 64 tokens and a head that a workgroup may take in a row before a sequence is cut at all: the pass that sums segments, the one
// that joins them and their launches cost about what these do.  One sequence, 8 heads of 64 in bf16, us replayed (called one by one), cut against
// whole: forward, 3 steps 12.9 (15.7) against 11.8 (12.2), 4 steps 13.2 (15.7) against 14.7 (15.2), 5 steps 13.4 (15.8) against 17.5 (18.0), 8 steps
// 14.1 (15.9) against 25.9 (26.4); the gradient, whose three sweeps repay the extra launches sooner, 2 steps 26.9 (29.0) against 22.9 (24.2), 3 steps
// 26.8 (29.0) against 29.7 (30.6) but 16 heads of 128 47.1 (49.3) against 38.8 (39.7), 4 steps 28.4 (30.2) against 36.5 (37.6).
constexpr int64_t kUncutSteps = 4, kUncutStepsBackward = 3;

// A launch has fewer than 2^32 threads; the step takes 1024 for a state of 128 x 128, the scan's kernels no more than 512 for one.
constexpr int64_t kMostStates = 1 << 22;
constexpr int kMostChannels8 = 1 << 20;

msla_status check_shape(const msla_recurrence* s, msla_dtype dt) {
    if (s == nullptr || !known(dt)) return MSLA_ERR_INVALID_ARG;
    if (s->sequences <= 0 || s->tokens < 0 || s->heads_q <= 0 || s->heads_kv <= 0 || s->head_dim <= 0) return MSLA_ERR_INVALID_ARG;
    if (s->heads_q % s->heads_kv != 0 || !(fabsf(s->scale) < INFINITY) || (s->rectify != 0 && s->rectify != 1)) return MSLA_ERR_INVALID_ARG;
    if (s->offsets == nullptr && s->tokens % s->sequences != 0) return MSLA_ERR_INVALID_ARG;
    if (s->offsets != nullptr && !aligned(s->offsets, 4)) return MSLA_ERR_INVALID_ARG;
    if (s->head_dim != 16 && s->head_dim != 32 && s->head_dim != 64 && s->head_dim != 128) return MSLA_ERR_UNSUPPORTED;
    if (s->heads_q > 32768 || s->tokens > 0x7fffffffLL || (int64_t)s->sequences * s->heads_kv >= kMostStates) return MSLA_ERR_UNSUPPORTED;
    return MSLA_OK;
}

int heads_per_group(const msla_recurrence& s) { return s.head_dim >= 64 ? 1 : 64 / s.head_dim; }       // state heads of a workgroup of the scan

// Segments are as long as leaves kWantGroups workgroups.  One that spans all tokens keeps every sequence whole.
msla_status plan_of(const msla_recurrence& s, bool backward, RecurrencePlan* plan) {
    const int per_group = heads_per_group(s);
    const int64_t groups = (s.heads_kv + per_group - 1) / per_group;
    const int64_t want = (kWantGroups + groups - 1) / groups;
    int64_t segment = (s.tokens / want + 63) / 64 * 64;
    const int64_t least = s.head_dim == 128 ? 128 : 64;         // (a state of 128 x 128 is as much traffic as four tiles of 64 tokens)
    if (segment < least) segment = least;
    const int64_t longest = s.offsets ? s.tokens : s.tokens / s.sequences;
    // (equal sequences that are workgroups enough for half of the places run whole: cut, they do 1.4 times the work)
    const bool enough = s.offsets == nullptr && s.sequences * groups * 2 >= kWantGroups;
    plan->cut = longest > segment && !enough && (longest + 63) / 64 * (s.heads_q / s.heads_kv) > (backward ? kUncutStepsBackward : kUncutSteps);
    if (!plan->cut) segment = (s.tokens / 64 + 1) * 64;
    const int64_t slots = s.tokens / segment + s.sequences;
    if (segment > 0x7fffffffLL || slots > 0x7fffffffLL / s.heads_kv) return MSLA_ERR_UNSUPPORTED;
    plan->segment = (int)segment;
    plan->slots = (int)slots;
    const size_t state = (size_t)s.head_dim * s.head_dim * 4, states = align_up((size_t)slots * s.heads_kv * state),
                 decays = align_up((size_t)slots * s.heads_kv * 4);
    size_t at = 0;
    if (plan->cut) {
        at = states;
        if (backward) {
            plan->d_states_at = at;
            at += states;
        }
        plan->decay_at = at;
        at += decays;
        if (backward) {
            plan->d_decay_at = at;
            at += decays;
            plan->crossing_at = at;
            at += decays * 16;          // (at most 16 parts of a state's 128 x 128 numbers)
        }
    }
    if (backward) {
        plan->dots_at = at;
        at += align_up((size_t)s.tokens * (s.heads_q + s.heads_kv) * 4);
        plan->last_at = at;
        at += align_up((size_t)s.sequences * s.heads_kv * state);
    }
    plan->bytes = at;
    return MSLA_OK;
}

// Strides that the kernels' 32-bit offsets inside a chunk of 64 tokens cover, in bytes.
constexpr int64_t kMostTokenStride = ((int64_t)1 << 24) - 1, kMostHeadStride = (int64_t)1 << 29;

bool wide(const msla_heads& h, msla_dtype dt) {
    const int64_t e = (int64_t)elem_size(dt);
    return h.token_stride * e > kMostTokenStride || h.head_stride * e > kMostHeadStride;
}

// ... and what such an offset reaches in an operand that a workgroup reads for all of its state heads, each with `heads / heads_kv` of the
// operand's: from the first one's first row to the last one's last, below the offset that stands for "not read" (2^32 - 16).
bool beyond_reach(const msla_heads& h, const msla_recurrence& s, int heads, msla_dtype dt) {
    if (s.tokens == 0) return false;
    const int64_t states = heads_per_group(s) < s.heads_kv ? heads_per_group(s) : s.heads_kv, rows = s.tokens < 64 ? s.tokens : 64;
    const int64_t last = (rows - 1) * h.token_stride + (states - 1) * (heads / s.heads_kv) * h.head_stride + s.head_dim;
    return last * (int64_t)elem_size(dt) > 0xfffffff0LL;
}

// a [tokens, heads, head_dim] operand: 16-byte pieces, no span beyond kMost
bool fits(const msla_heads& h, const msla_recurrence& s, int heads, msla_dtype dt) {
    if (s.tokens == 0) return true;
    const int64_t unit = (int64_t)(16 / elem_size(dt));
    if (h.data == nullptr || !aligned(h.data, 16) || h.token_stride < 0 || h.head_stride < 0) return false;
    if (h.token_stride % unit != 0 || h.head_stride % unit != 0) return false;
    if (h.token_stride > kMost / s.tokens || h.head_stride > kMost / heads) return false;
    return true;
}

// ... that is written: its rows lie apart
bool apart(const msla_heads& h, const msla_recurrence& s, int heads) {
    if (s.tokens == 0) return true;
    const int64_t d = s.head_dim, n = s.tokens;
    const bool by_token = (heads == 1 || h.head_stride >= d) && (n == 1 || h.token_stride >= (heads - 1) * h.head_stride + d);
    const bool by_head = (n == 1 || h.token_stride >= d) && (heads == 1 || h.head_stride >= (n - 1) * h.token_stride + d);
    return by_token || by_head;
}

bool gate_fits(const void* gate, int64_t stride, const msla_recurrence& s, msla_dtype dt, bool written) {
    if (gate == nullptr || s.tokens == 0) return true;
    if (!aligned(gate, elem_size(dt)) || stride < 0 || stride * (int64_t)elem_size(dt) > kMostTokenStride) return false;
    return !written || s.tokens == 1 || stride >= s.heads_kv;
}

RecurrenceRows rows_of(const msla_heads& h) { return RecurrenceRows{h.data, (long)h.token_stride, (long)h.head_stride}; }

void fill(RecurrenceCall* c, const msla_recurrence& s, const msla_heads& q, const msla_heads& k, const msla_heads& v, const void* gate,
          int64_t gate_stride, const float* initial) {
    c->sequences = s.sequences;
    c->tokens = (long)s.tokens;
    c->offsets = s.offsets;
    c->heads_q = s.heads_q;
    c->heads_kv = s.heads_kv;
    c->head_dim = s.head_dim;
    c->rectify = s.rectify;
    c->scale = s.scale;
    c->q = rows_of(q);
    c->k = rows_of(k);
    c->v = rows_of(v);
    c->gate = gate;
    c->gate_ts = (long)gate_stride;
    c->initial = initial;
}

bool same(const msla_heads& out, const msla_heads& in) { return out.data != nullptr && out.data == in.data; }

}  // namespace

extern "C" {

msla_status msla_recurrence_workspace_bytes(const msla_recurrence* shape, int backward, msla_dtype dt, size_t* bytes) {
    if (bytes == nullptr) return MSLA_ERR_INVALID_ARG;
    msla_status st = check_shape(shape, dt);
    if (st != MSLA_OK) return st;
    RecurrencePlan plan;
    st = plan_of(*shape, backward != 0, &plan);
    if (st == MSLA_OK) *bytes = plan.bytes;
    return st;
}

msla_status msla_recurrence_forward(const msla_recurrence* shape, msla_heads q, msla_heads k, msla_heads v, const void* log_gate,
                                    int64_t gate_stride, const float* initial_state, msla_heads out, float* final_state, void* workspace,
                                    size_t workspace_bytes, msla_dtype dt, void* stream) {
    msla_status st = check_shape(shape, dt);
    if (st != MSLA_OK) return st;
    const msla_recurrence& s = *shape;
    if (!fits(q, s, s.heads_q, dt) || !fits(k, s, s.heads_kv, dt) || !fits(v, s, s.heads_kv, dt) || !fits(out, s, s.heads_q, dt) ||
        !apart(out, s, s.heads_q) || !gate_fits(log_gate, gate_stride, s, dt, false) || !aligned(initial_state, 16) ||
        !aligned(final_state, 16) || same(out, q) || same(out, k) || same(out, v))
        return MSLA_ERR_INVALID_ARG;
    if (wide(q, dt) || wide(k, dt) || wide(v, dt) || wide(out, dt) || beyond_reach(q, s, s.heads_q, dt)) return MSLA_ERR_UNSUPPORTED;
    RecurrenceCall c = {};
    st = plan_of(s, false, &c.plan);
    if (st != MSLA_OK) return st;
    if (c.plan.bytes > 0 && (workspace == nullptr || !aligned(workspace, 16))) return MSLA_ERR_INVALID_ARG;
    if (workspace_bytes < c.plan.bytes) return MSLA_ERR_WORKSPACE;
    fill(&c, s, q, k, v, log_gate, gate_stride, initial_state);
    c.what = 0;
    c.out = rows_of(out);
    c.final_state = final_state;
    c.ws = (char*)workspace;
    return status_of(msla::launch_recurrence((int)dt, c, (hipStream_t)stream));
}

msla_status msla_recurrence_backward(const msla_recurrence* shape, msla_heads q, msla_heads k, msla_heads v, const void* log_gate,
                                     int64_t gate_stride, const float* initial_state, msla_heads d_out, const float* d_final_state,
                                     msla_heads d_q, msla_heads d_k, msla_heads d_v, void* d_log_gate, int64_t d_gate_stride,
                                     float* d_initial_state, void* workspace, size_t workspace_bytes, msla_dtype dt, void* stream) {
    msla_status st = check_shape(shape, dt);
    if (st != MSLA_OK) return st;
    const msla_recurrence& s = *shape;
    if (!fits(q, s, s.heads_q, dt) || !fits(k, s, s.heads_kv, dt) || !fits(v, s, s.heads_kv, dt) || !fits(d_out, s, s.heads_q, dt) ||
        !fits(d_q, s, s.heads_q, dt) || !fits(d_k, s, s.heads_kv, dt) || !fits(d_v, s, s.heads_kv, dt) || !apart(d_q, s, s.heads_q) ||
        !apart(d_k, s, s.heads_kv) || !apart(d_v, s, s.heads_kv) || !gate_fits(log_gate, gate_stride, s, dt, false) ||
        !gate_fits(d_log_gate, d_gate_stride, s, dt, true) || !aligned(initial_state, 16) || !aligned(d_final_state, 16) ||
        !aligned(d_initial_state, 16))
        return MSLA_ERR_INVALID_ARG;
    if (d_log_gate != nullptr && log_gate == nullptr) return MSLA_ERR_INVALID_ARG;
    if (d_initial_state != nullptr && (d_initial_state == d_final_state || d_initial_state == initial_state)) return MSLA_ERR_INVALID_ARG;
    for (const msla_heads* o : {&d_q, &d_k, &d_v})
        for (const msla_heads* i : {&q, &k, &v, &d_out})
            if (same(*o, *i)) return MSLA_ERR_INVALID_ARG;
    if (same(d_q, d_k) || same(d_q, d_v) || same(d_k, d_v)) return MSLA_ERR_INVALID_ARG;
    for (const msla_heads* h : {&q, &k, &v, &d_out, &d_q, &d_k, &d_v})
        if (wide(*h, dt)) return MSLA_ERR_UNSUPPORTED;
    if (beyond_reach(q, s, s.heads_q, dt) || beyond_reach(d_out, s, s.heads_q, dt)) return MSLA_ERR_UNSUPPORTED;
    RecurrenceCall c = {};
    st = plan_of(s, true, &c.plan);
    if (st != MSLA_OK) return st;
    if (workspace == nullptr || !aligned(workspace, 16)) return MSLA_ERR_INVALID_ARG;
    if (workspace_bytes < c.plan.bytes) return MSLA_ERR_WORKSPACE;
    fill(&c, s, q, k, v, log_gate, gate_stride, initial_state);
    c.what = 1;
    c.d_out = rows_of(d_out);
    c.d_final = d_final_state;
    c.d_q = rows_of(d_q);
    c.d_k = rows_of(d_k);
    c.d_v = rows_of(d_v);
    c.d_gate = d_log_gate;
    c.d_gate_ts = (long)d_gate_stride;
    c.d_initial = d_initial_state;
    c.ws = (char*)workspace;
    return status_of(msla::launch_recurrence((int)dt, c, (hipStream_t)stream));
}

msla_status msla_recurrence_step(const msla_recurrence* shape, msla_heads q, msla_heads k, msla_heads v, const void* log_gate,
                                 int64_t gate_stride, const float* state, msla_heads out, float* new_state, msla_dtype dt, void* stream) {
    msla_status st = check_shape(shape, dt);
    if (st != MSLA_OK) return st;
    const msla_recurrence& s = *shape;
    if (s.offsets != nullptr || s.tokens != s.sequences || new_state == nullptr) return MSLA_ERR_INVALID_ARG;
    if (!fits(q, s, s.heads_q, dt) || !fits(k, s, s.heads_kv, dt) || !fits(v, s, s.heads_kv, dt) || !fits(out, s, s.heads_q, dt) ||
        !apart(out, s, s.heads_q) || !gate_fits(log_gate, gate_stride, s, dt, false) || !aligned(state, 16) || !aligned(new_state, 16) ||
        same(out, q) || same(out, k) || same(out, v))
        return MSLA_ERR_INVALID_ARG;
    if (wide(q, dt) || wide(k, dt) || wide(v, dt) || wide(out, dt)) return MSLA_ERR_UNSUPPORTED;
    RecurrenceCall c = {};
    fill(&c, s, q, k, v, log_gate, gate_stride, state);
    c.what = 2;
    c.out = rows_of(out);
    c.final_state = new_state;
    return status_of(msla::launch_recurrence((int)dt, c, (hipStream_t)stream));
}

static msla_status check_rows(int64_t rows, int channels, float eps, msla_dtype dt) {
    if (rows < 0 || channels <= 0 || !(eps >= 0.0f) || !(eps < INFINITY) || !known(dt)) return MSLA_ERR_INVALID_ARG;
    if (channels > 32768 || rows > 0x7fffffffLL) return MSLA_ERR_UNSUPPORTED;
    return MSLA_OK;
}

static msla_status norm(const void* x, const void* residual, const void* weight, void* y, float* scale, bool eight, bool plain, void* sum,
                        int64_t rows, int channels, float eps, msla_dtype dt, void* stream) {
    const msla_status st = check_rows(rows, channels, eps, dt);
    if (st != MSLA_OK) return st;
    const size_t e = elem_size(dt);
    if (!aligned(x, e) || !aligned(residual, e) || !aligned(weight, e) || !aligned(sum, e) || !aligned(y, eight ? 1 : e) || !aligned(scale, 4))
        return MSLA_ERR_INVALID_ARG;
    if (rows == 0) return MSLA_OK;
    if (x == nullptr || y == nullptr || (eight && (scale == nullptr || y == x))) return MSLA_ERR_INVALID_ARG;
    if (y == sum || (residual != nullptr && y == residual)) return MSLA_ERR_INVALID_ARG;
    const NormCall c = {x, residual, weight, y, sum, scale, rows, channels, eps, plain};
    return status_of(msla::launch_norm((int)dt, c, (hipStream_t)stream));
}

msla_status msla_norm_forward(const void* x, const void* residual, const void* weight, void* y, void* sum, int64_t rows, int channels, float eps,
                              msla_dtype dt, void* stream) {
    return norm(x, residual, weight, y, nullptr, false, false, sum, rows, channels, eps, dt, stream);
}

msla_status msla_norm_quantized(const void* x, const void* residual, const void* weight, void* y8, float* scale, void* sum, int64_t rows,
                                int channels, float eps, msla_dtype dt, void* stream) {
    return norm(x, residual, weight, y8, scale, true, false, sum, rows, channels, eps, dt, stream);
}

msla_status msla_quantize_rows(const void* x, void* x8, float* scale, int64_t rows, int channels, msla_dtype dt, void* stream) {
    return norm(x, nullptr, nullptr, x8, scale, true, true, nullptr, rows, channels, 0.0f, dt, stream);
}

msla_status msla_norm_backward_workspace_bytes(int64_t rows, int channels, msla_dtype dt, size_t* bytes) {
    if (bytes == nullptr) return MSLA_ERR_INVALID_ARG;
    const msla_status st = check_rows(rows, channels, 0.0f, dt);
    if (st == MSLA_OK) *bytes = align_up((size_t)msla::norm_backward_blocks(rows, channels, (int)elem_size(dt)) * channels * 4);
    return st;
}

msla_status msla_norm_backward(const void* sum, const void* weight, const void* d_y, const void* d_sum, void* d_r, float* d_weight,
                               void* workspace, size_t workspace_bytes, int64_t rows, int channels, float eps, msla_dtype dt, void* stream) {
    const msla_status st = check_rows(rows, channels, eps, dt);
    if (st != MSLA_OK) return st;
    const size_t e = elem_size(dt);
    if (!aligned(sum, e) || !aligned(weight, e) || !aligned(d_y, e) || !aligned(d_sum, e) || !aligned(d_r, e) || !aligned(d_weight, 4))
        return MSLA_ERR_INVALID_ARG;
    if (rows > 0 && (sum == nullptr || d_y == nullptr || d_r == nullptr || d_r == sum)) return MSLA_ERR_INVALID_ARG;
    if (d_weight != nullptr && rows > 0) {
        if (workspace == nullptr || !aligned(workspace, 16)) return MSLA_ERR_INVALID_ARG;
        if (workspace_bytes < (size_t)msla::norm_backward_blocks(rows, channels, (int)e) * channels * 4) return MSLA_ERR_WORKSPACE;
    }
    return status_of(msla::launch_norm_backward((int)dt, sum, weight, d_y, d_sum, d_r, d_weight, (float*)workspace, rows, channels, eps,
                                                (hipStream_t)stream));
}

msla_status msla_linear_quantized(const void* x8, const float* x_scale, const void* w8, const float* w_scale, void* y, int64_t rows, int c_in,
                                  int c_out, msla_dtype dt, void* stream) {
    if (rows < 0 || c_in <= 0 || c_out <= 0 || !known(dt)) return MSLA_ERR_INVALID_ARG;
    if (!aligned(x8, 16) || !aligned(w8, 16) || !aligned(y, 16) || !aligned(x_scale, 4) || !aligned(w_scale, 4)) return MSLA_ERR_INVALID_ARG;
    if (c_in % 16 != 0 || c_out % 16 != 0 || c_in > kMostChannels8 || c_out > kMostChannels8 || rows > 0x7fffffffLL) return MSLA_ERR_UNSUPPORTED;
    if (rows == 0) return MSLA_OK;
    if (!x8 || !x_scale || !w8 || !w_scale || !y || y == x8 || y == w8) return MSLA_ERR_INVALID_ARG;
    return status_of(msla::launch_linear_quantized((int)dt, x8, x_scale, w8, w_scale, y, rows, c_in, c_out, (hipStream_t)stream));
}

}  // extern "C"
