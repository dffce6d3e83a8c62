// C ABI of the operators beside the attention: argument checks and launches.  Nothing here touches tensor data.
#include <math.h>

#include "../../include/leet_attn.h"
#include "leet_gated_scan.hpp"
#include "leet_heads.hpp"
#include "leet_host.hpp"
#include "leet_overlap.hpp"

namespace {

using leet::Dim;
using leet::Span;

// A launch has fewer than 2^32 threads.
constexpr long long kMaxThreads = 1LL << 32;
// Sums of heads, and of sequences, stay within an int.
constexpr int kMaxHeads = 1 << 28, kMaxSequences = 1 << 30;

int elem_of(int dtype) { return dtype == LEET_F32 ? 0 : dtype == LEET_BF16 ? 1 : 2; }
bool dtype_ok(int dtype) { return dtype == LEET_F32 || dtype == LEET_BF16 || dtype == LEET_F16; }
size_t size_of(int dtype) { return dtype == LEET_F32 ? 4 : 2; }
bool aligned(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

// Whether rows of `width` adjacent elements at these strides cannot overlap (checked from the smallest stride up, which
// every layout of a dense tensor and of a part of one passes).
bool rows_apart(long long width, Dim* dims, int n) {
    for (int i = 0; i < n; ++i)
        for (int j = i + 1; j < n; ++j)
            if (dims[j].stride < dims[i].stride) {
                const Dim t = dims[i];
                dims[i] = dims[j];
                dims[j] = t;
            }
    long long extent = width;
    for (int i = 0; i < n; ++i) {
        if (dims[i].size <= 1) continue;
        if (dims[i].stride < extent) return false;
        extent += (dims[i].size - 1) * dims[i].stride;
    }
    return true;
}

bool shares_any(const Span& out, std::initializer_list<const Span*> others) {
    for (const Span* o : others)
        if (overlap(out, *o)) return true;
    return false;
}

// ---- heads ----

// Rows read and written beyond this are streamed past the last-level cache (256 MiB, 0.6 of it: where the prefill's inputs
// begin to fall out of it too).  us with and without, forward B4 H16+16 d128 bf16, the same tensors again and again |
// four sets in turn: N 2048 (128 MiB in and out) 29 23 | 29 34, N 2816 (176 MiB) 38 33 | 39 48, N 4096 51 52 | 52 63,
// N 6144 75 88 | 75 88.
constexpr size_t kStreamBytes = ((size_t)256 << 20) / 5 * 3;

bool heads_ok(const leet_attn_heads* t, int B, int H, int N, int d, size_t size, bool written) {
    if (!t || !t->data || !aligned(t->data, size)) return false;
    Dim dims[3] = {{B, t->batch}, {H, t->head}, {N, t->token}};
    return !written || rows_apart(d, dims, 3);
}

Span span_of(const leet_attn_heads* t, int B, int H, int N, int d, long long size) {
    return t ? Span(t->data, size, d, {{B, t->batch}, {H, t->head}, {N, t->token}}) : Span();
}
// Whether an output is its input, stride for stride, or apart from it.
bool in_place_or_apart(const Span& out, const Span& in) { return out == in || !overlap(out, in); }

struct HeadsCall {
    const leet_attn_heads *in, *grad, *out;
    int H;
    const void* weight;
    void* weight_grad;
};

// The arguments that the three operators on heads share.  LEET_OK with p->tokens = 0: nothing to do.
// workspace: of the backward pass.
int heads_params(const HeadsCall& q, const HeadsCall& k, const leet_attn_rotation* rotation, bool keys, bool backward,
                 int weight_dtype, float eps, const void* workspace, int B, int N, int d, int dtype, leet::HeadsParams* p) {
    if (!rotation || B <= 0 || N < 0 || q.H <= 0 || (keys && k.H <= 0)) return LEET_ERR_INVALID_ARG;
    if (!dtype_ok(dtype) || (weight_dtype != LEET_F32 && weight_dtype != dtype)) return LEET_ERR_UNSUPPORTED;
    if (d < 2 || d > 256 || d % 2 != 0) return LEET_ERR_UNSUPPORTED;
    if (!rotation->freq || !aligned(rotation->freq, 8) || !aligned(rotation->positions, 8)) return LEET_ERR_INVALID_ARG;
    if (rotation->rot < 2 || rotation->rot > d || rotation->rot % 2 != 0) return LEET_ERR_INVALID_ARG;
    if (rotation->layout != LEET_ROPE_HALF && rotation->layout != LEET_ROPE_INTERLEAVED) return LEET_ERR_INVALID_ARG;
    if (!isfinite(rotation->scale) || !isfinite(eps) || eps < 0.0f) return LEET_ERR_INVALID_ARG;
    if ((long long)B * N >= 1LL << 31 || q.H > kMaxHeads || (keys && k.H > kMaxHeads)) return LEET_ERR_TOO_LARGE;
    *p = leet::HeadsParams{};
    p->tokens = B * N;
    if (N == 0) return LEET_OK;
    const size_t size = size_of(dtype), weight_size = size_of(weight_dtype);
    p->vector = d % 8 == 0 && (rotation->layout == LEET_ROPE_INTERLEAVED || rotation->rot % 8 == 0);
    p->stream = (size_t)B * N * (q.H + (keys ? k.H : 0)) * d * size * (backward ? 3 : 2) > kStreamBytes;
    for (const HeadsCall* c : {&q, &k}) {
        if (c == &k && !keys) continue;
        if (!heads_ok(c->in, B, c->H, N, d, size, false) ||
            !heads_ok(c->out, B, c->H, N, d, size, true) ||
            (backward && !heads_ok(c->grad, B, c->H, N, d, size, false)))
            return LEET_ERR_INVALID_ARG;
        if (!aligned(c->weight, weight_size) || !aligned(c->weight_grad, weight_size)) return LEET_ERR_INVALID_ARG;
        leet::HeadRows& r = c == &q ? p->q : p->k;
        r.in = static_cast<const char*>(c->in->data);
        r.in_b = c->in->batch; r.in_h = c->in->head; r.in_n = c->in->token;
        r.out = static_cast<char*>(c->out->data);
        r.out_b = c->out->batch; r.out_h = c->out->head; r.out_n = c->out->token;
        if (backward) {
            r.grad = static_cast<const char*>(c->grad->data);
            r.grad_b = c->grad->batch; r.grad_h = c->grad->head; r.grad_n = c->grad->token;
        }
        r.weight = c->weight;
        r.weight_grad = c->weight_grad;
        r.H = c->H;
    }
    p->freq = rotation->freq;
    p->positions = rotation->positions;
    p->positions_batch = rotation->positions_batch;
    p->pos0 = rotation->pos0;
    p->scale = rotation->scale;
    p->rot = rotation->rot;
    p->eps = eps;
    p->d = d;
    p->N = N;
    p->weight_f32 = weight_dtype == LEET_F32;
    leet::plan_heads(p, backward);
    // a wave takes 64 lanes of tokens of at least one lane each, for one unit
    if ((long long)p->tokens * p->units * 64 >= kMaxThreads) return LEET_ERR_TOO_LARGE;
    // an output may be what it is made from; everything else that is written lies apart from the rest
    const long long isz = (long long)size, wsz = (long long)weight_size;
    const Span q_in = span_of(q.in, B, q.H, N, d, isz), q_out = span_of(q.out, B, q.H, N, d, isz);
    const Span k_in = span_of(k.in, B, k.H, N, d, isz), k_out = span_of(k.out, B, k.H, N, d, isz);
    const Span q_grad = span_of(q.grad, B, q.H, N, d, isz), k_grad = span_of(k.grad, B, k.H, N, d, isz);
    const Span q_weight(q.weight, wsz, d), k_weight(k.weight, wsz, d), freq(rotation->freq, 8, rotation->rot / 2);
    const Span positions(rotation->positions, 8, N, {{B, rotation->positions_batch}});
    if (!in_place_or_apart(q_out, q_in) || !in_place_or_apart(q_out, q_grad) || !in_place_or_apart(k_out, k_in) ||
        !in_place_or_apart(k_out, k_grad) ||
        shares_any(q_out, {&k_out, &k_in, &k_grad, &q_weight, &k_weight, &freq, &positions}) ||
        shares_any(k_out, {&q_in, &q_grad, &q_weight, &k_weight, &freq, &positions}))
        return LEET_ERR_INVALID_ARG;
    if (backward) {
        const Span q_sum(q.weight_grad, wsz, d), k_sum(k.weight_grad, wsz, d);
        // written when all else has been read
        if (shares_any(q_sum, {&k_sum, &q_out, &k_out}) || shares_any(k_sum, {&q_out, &k_out})) return LEET_ERR_INVALID_ARG;
        if (q.weight_grad || k.weight_grad) {
            const Span scratch(workspace, sizeof(float), (long long)p->groups * p->units * d);
            if (shares_any(scratch, {&q_out, &k_out, &q_in, &k_in, &q_grad, &k_grad, &q_weight, &k_weight, &freq, &positions,
                                     &q_sum, &k_sum}))
                return LEET_ERR_INVALID_ARG;
        }
    }
    int dev = 0;
    return leet::current_device(&dev);
}

int done(hipError_t e) { return e == hipSuccess ? LEET_OK : LEET_ERR_LAUNCH; }

// ---- gated scan ----

bool rows_ok(const leet_attn_rows* t, int B, int N, int C, size_t size, bool written) {
    if (!t || !t->data || !aligned(t->data, size)) return false;
    Dim dims[2] = {{B, t->batch}, {N, t->token}};
    return !written || rows_apart(C, dims, 2);
}
Span span_of(const leet_attn_rows* t, int B, int N, int C, long long size) {
    return t ? Span(t->data, size, C, {{B, t->batch}, {N, t->token}}) : Span();
}
Span states_of(const float* s, int S, int C) { return Span(s, 4, (long long)S * C); }
// Whether rows can be taken four channels at a time.
bool by_four(const leet_attn_rows* t, int B, size_t size) {
    return aligned(t->data, 4 * size) && (B <= 1 || t->batch % 4 == 0);
}

leet::RowsIn rows_in(const leet_attn_rows* t) { return {static_cast<const char*>(t->data), t->batch, t->token}; }
leet::RowsOut rows_out(const leet_attn_rows* t) { return {static_cast<char*>(t->data), t->batch, t->token}; }

int scan_types_ok(int dtype, int gate_dtype, int mode) {
    if (mode != LEET_GATE_DECAY && mode != LEET_GATE_LOG && mode != LEET_GATE_SIGMOID) return LEET_ERR_INVALID_ARG;
    return dtype_ok(dtype) && (gate_dtype == dtype || gate_dtype == LEET_F32) ? LEET_OK : LEET_ERR_UNSUPPORTED;
}

// Sizes, offsets and workspace of a call over whole sequences; *S receives the number of sequences.
int scan_sizes_ok(const int* offsets, int sequences, const void* workspace, size_t workspace_bytes, int B, int N, int C,
                  int backward, int* S) {
    if (B <= 0 || N < 0 || C <= 0) return LEET_ERR_INVALID_ARG;
    if (offsets && (B != 1 || sequences < 0 || !aligned(offsets, 4))) return LEET_ERR_INVALID_ARG;
    if (N > 1 << 30 || C > 1 << 28 || (offsets && sequences > kMaxSequences) ||
        leet::gated_scan_threads(B, N, C, backward != 0) >= kMaxThreads)
        return LEET_ERR_TOO_LARGE;
    const size_t need = leet_attn_gated_scan_workspace_bytes(B, N, C, backward);
    if (need && (!workspace || workspace_bytes < need || !aligned(workspace, 256))) return LEET_ERR_INVALID_ARG;
    *S = offsets ? sequences : B;
    return LEET_OK;
}

}  // namespace

extern "C" {

int leet_attn_rope_frequencies(int rot, double base, int scaling, double factor, int trained, double slow,
                               double fast, double *freq, float *scale) {
    if (rot < 2 || rot % 2 != 0 || !(base > 1.0) || !isfinite(base) || !(factor >= 1.0) || !isfinite(factor) || !freq ||
        !scale || scaling < LEET_ROPE_SCALING_NONE || scaling > LEET_ROPE_SCALING_TURNS)
        return LEET_ERR_INVALID_ARG;
    const bool ends = scaling == LEET_ROPE_SCALING_BANDS || scaling == LEET_ROPE_SCALING_TURNS;
    if (ends && (trained <= 0 || !(slow > 0.0) || !(fast > slow) || !isfinite(fast))) return LEET_ERR_INVALID_ARG;
    const double kTwoPi = 6.283185307179586476925;
    if (scaling == LEET_ROPE_SCALING_BASE && rot > 2) base *= pow(factor, rot / (rot - 2.0));
    // the pair (not whole) that turns so many times within the trained length
    auto index = [&](double turns) { return rot * log(trained / (turns * kTwoPi)) / (2.0 * log(base)); };
    const double low = ends ? fmax(floor(index(fast)), 0.0) : 0.0;
    const double high = ends ? fmin(ceil(index(slow)), rot - 1.0) : 0.0;
    for (int i = 0; i < rot / 2; ++i) {
        const double f = pow(base, -2.0 * i / rot);
        double stretched = 0.0;  // share of the frequency divided by the factor
        if (scaling == LEET_ROPE_SCALING_LINEAR) stretched = 1.0;
        else if (scaling == LEET_ROPE_SCALING_BANDS) stretched = (i - low) / fmax(high - low, 1e-3);
        else if (scaling == LEET_ROPE_SCALING_TURNS) stretched = (fast - trained * f / kTwoPi) / (fast - slow);
        stretched = fmin(fmax(stretched, 0.0), 1.0);
        freq[i] = stretched == 1.0 ? f / factor : f * (1.0 - stretched) + f / factor * stretched;
    }
    *scale = scaling == LEET_ROPE_SCALING_BANDS ? (float)(0.1 * log(factor) + 1.0) : 1.0f;
    return LEET_OK;
}

int leet_attn_rope(const leet_attn_heads *q, const leet_attn_heads *out_q, int Hq,
                   const leet_attn_heads *k, const leet_attn_heads *out_k, int Hk,
                   const leet_attn_rotation *rotation, int B, int N, int d, int dtype, int transposed,
                   void *stream) {
    if (!k != !out_k) return LEET_ERR_INVALID_ARG;
    leet::HeadsParams p;
    const int status = heads_params({q, nullptr, out_q, Hq, nullptr, nullptr}, {k, nullptr, out_k, Hk, nullptr, nullptr},
                                    rotation, k != nullptr, false, dtype, 0.0f, nullptr, B, N, d, dtype, &p);
    if (status != LEET_OK || p.tokens == 0) return status;
    p.transposed = transposed != 0;
    return done(leet::launch_heads(p, elem_of(dtype), rotation->layout, false, static_cast<hipStream_t>(stream)));
}

int leet_attn_qk_norm_rope(const leet_attn_heads *q, const leet_attn_heads *out_q, int Hq,
                           const leet_attn_heads *k, const leet_attn_heads *out_k, int Hk,
                           const void *q_weight, const void *k_weight, int weight_dtype, float eps,
                           const leet_attn_rotation *rotation, int B, int N, int d, int dtype, void *stream) {
    leet::HeadsParams p;
    const int status = heads_params({q, nullptr, out_q, Hq, q_weight, nullptr}, {k, nullptr, out_k, Hk, k_weight, nullptr},
                                    rotation, true, false, weight_dtype, eps, nullptr, B, N, d, dtype, &p);
    if (status != LEET_OK || p.tokens == 0) return status;
    return done(leet::launch_heads(p, elem_of(dtype), rotation->layout, true, static_cast<hipStream_t>(stream)));
}

size_t leet_attn_qk_norm_rope_workspace_bytes(int B, int Hq, int Hk, int N, int d) {
    if (B <= 0 || Hq <= 0 || Hk <= 0 || N <= 0 || d < 2 || d > 256 || d % 2 != 0 || (long long)B * N >= 1LL << 31 ||
        Hq > kMaxHeads || Hk > kMaxHeads)
        return 0;
    // the cuts of rows and their way from memory give different numbers of workgroups; room for any
    size_t rows = 0;
    for (int way = 0; way < 4; ++way) {
        leet::HeadsParams p = {};
        p.q.H = Hq;
        p.k.H = Hk;
        p.tokens = B * N;
        p.d = d;
        p.vector = way & 1;
        p.stream = way >> 1;
        leet::plan_heads(&p, true);
        const size_t r = (size_t)p.groups * p.units;
        if (r > rows) rows = r;
    }
    return rows * d * sizeof(float);
}

int leet_attn_qk_norm_rope_backward(const leet_attn_heads *dout_q, const leet_attn_heads *q,
                                    const leet_attn_heads *dq, int Hq,
                                    const leet_attn_heads *dout_k, const leet_attn_heads *k,
                                    const leet_attn_heads *dk, int Hk,
                                    const void *q_weight, const void *k_weight, void *dq_weight, void *dk_weight,
                                    int weight_dtype, float eps, const leet_attn_rotation *rotation,
                                    void *workspace, size_t workspace_bytes,
                                    int B, int N, int d, int dtype, void *stream) {
    leet::HeadsParams p;
    const int status = heads_params({q, dout_q, dq, Hq, q_weight, dq_weight}, {k, dout_k, dk, Hk, k_weight, dk_weight},
                                    rotation, true, true, weight_dtype, eps, workspace, B, N, d, dtype, &p);
    if (status != LEET_OK) return status;
    const bool sums = dq_weight || dk_weight;
    if (p.tokens == 0) {
        // no tokens: the sums are empty, and still they are outputs
        if (!sums) return LEET_OK;
        if (!aligned(dq_weight, size_of(weight_dtype)) || !aligned(dk_weight, size_of(weight_dtype))) return LEET_ERR_INVALID_ARG;
        int dev = 0;
        const int found = leet::current_device(&dev);
        if (found != LEET_OK) return found;
        p.q.weight_grad = dq_weight;
        p.k.weight_grad = dk_weight;
        p.d = d;
        p.weight_f32 = weight_dtype == LEET_F32;
        return done(leet::launch_heads_weights(p, elem_of(dtype), static_cast<hipStream_t>(stream)));
    }
    if (sums) {
        if (!workspace || !aligned(workspace, 256) || workspace_bytes < (size_t)p.groups * p.units * d * sizeof(float))
            return LEET_ERR_INVALID_ARG;
        p.partial = static_cast<float*>(workspace);
    }
    hipError_t e = leet::launch_heads_backward(p, elem_of(dtype), rotation->layout, static_cast<hipStream_t>(stream));
    if (e == hipSuccess && sums) e = leet::launch_heads_weights(p, elem_of(dtype), static_cast<hipStream_t>(stream));
    return done(e);
}

size_t leet_attn_gated_scan_workspace_bytes(int B, int N, int C, int backward) {
    if (B <= 0 || N <= 0 || C <= 0 || N > 1 << 30 || C > 1 << 28 ||
        leet::gated_scan_threads(B, N, C, backward != 0) >= kMaxThreads)
        return 0;
    return leet::gated_scan_workspace(B, N, C, backward != 0);
}

int leet_attn_gated_scan(const leet_attn_rows *x, const leet_attn_rows *gate, const leet_attn_rows *out,
                         const float *state_in, float *state_out, const int *offsets, int sequences,
                         void *workspace, size_t workspace_bytes,
                         int B, int N, int C, int dtype, int gate_dtype, int mode, void *stream) {
    int status = scan_types_ok(dtype, gate_dtype, mode), S = 0;
    if (status == LEET_OK) status = scan_sizes_ok(offsets, sequences, workspace, workspace_bytes, B, N, C, 0, &S);
    if (status != LEET_OK) return status;
    leet::GatedScanParams p = {};
    if (N > 0) {
        if (!rows_ok(x, B, N, C, size_of(dtype), false) ||
            !rows_ok(gate, B, N, C, size_of(gate_dtype), false) ||
            !rows_ok(out, B, N, C, size_of(dtype), true))
            return LEET_ERR_INVALID_ARG;
        p.x = rows_in(x);
        p.gate = rows_in(gate);
        p.out = rows_out(out);
    }
    if (!aligned(state_in, 4) || !aligned(state_out, 4)) return LEET_ERR_INVALID_ARG;
    {
        const long long size = (long long)size_of(dtype);
        const Span rows_x = span_of(x, B, N, C, size), rows_gate = span_of(gate, B, N, C, (long long)size_of(gate_dtype));
        const Span to = span_of(out, B, N, C, size), in = states_of(state_in, S, C), left = states_of(state_out, S, C);
        const Span places(offsets, 4, S + 1LL), scratch(workspace, 1, (long long)leet_attn_gated_scan_workspace_bytes(B, N, C, 0));
        if (shares_any(to, {&rows_x, &rows_gate, &in, &left, &places, &scratch}) ||
            shares_any(left, {&rows_x, &rows_gate, &places, &scratch}) || (state_out != state_in && overlap(left, in)) ||
            shares_any(scratch, {&rows_x, &rows_gate, &in, &places}))
            return LEET_ERR_INVALID_ARG;
    }
    if (S == 0 || (N == 0 && (!state_out || state_out == state_in))) return LEET_OK;
    p.state_in = state_in;
    p.state_out = state_out;
    p.offsets = offsets;
    p.sequences = S;
    p.B = B; p.N = N; p.C = C;
    p.workspace = workspace;
    int dev = 0;
    status = leet::current_device(&dev);
    if (status != LEET_OK) return status;
    return done(leet::launch_gated_scan(p, elem_of(dtype), elem_of(gate_dtype), mode, static_cast<hipStream_t>(stream)));
}

int leet_attn_gated_scan_backward(const leet_attn_rows *dh, const leet_attn_rows *x, const leet_attn_rows *gate,
                                  const leet_attn_rows *h, const leet_attn_rows *dx, const leet_attn_rows *dgate,
                                  const float *state_in, const float *dstate_out, float *dstate_in,
                                  const int *offsets, int sequences, void *workspace, size_t workspace_bytes,
                                  int B, int N, int C, int dtype, int gate_dtype, int mode, void *stream) {
    int status = scan_types_ok(dtype, gate_dtype, mode), S = 0;
    if (status == LEET_OK) status = scan_sizes_ok(offsets, sequences, workspace, workspace_bytes, B, N, C, 1, &S);
    if (status != LEET_OK) return status;
    leet::GatedScanParams p = {};
    if (N > 0) {
        const size_t size = size_of(dtype), gate_size = size_of(gate_dtype);
        if (!rows_ok(dh, B, N, C, size, false) || !rows_ok(gate, B, N, C, gate_size, false) ||
            !rows_ok(h, B, N, C, size, false) || !rows_ok(dx, B, N, C, size, true) ||
            !rows_ok(dgate, B, N, C, gate_size, true))
            return LEET_ERR_INVALID_ARG;
        if (mode == LEET_GATE_SIGMOID) {
            if (!rows_ok(x, B, N, C, size, false)) return LEET_ERR_INVALID_ARG;
            p.x = rows_in(x);
        }
        p.dh = rows_in(dh);
        p.gate = rows_in(gate);
        p.h = rows_in(h);
        p.dx = rows_out(dx);
        p.dgate = rows_out(dgate);
    }
    if (!aligned(state_in, 4) || !aligned(dstate_out, 4) || !aligned(dstate_in, 4)) return LEET_ERR_INVALID_ARG;
    {
        const long long size = (long long)size_of(dtype), gate_size = (long long)size_of(gate_dtype);
        const Span rows_dh = span_of(dh, B, N, C, size), rows_gate = span_of(gate, B, N, C, gate_size);
        const Span rows_h = span_of(h, B, N, C, size), rows_x = p.x.data ? span_of(x, B, N, C, size) : Span();
        const Span to_x = span_of(dx, B, N, C, size), to_gate = span_of(dgate, B, N, C, gate_size);
        const Span in = states_of(state_in, S, C), behind = states_of(dstate_out, S, C), before = states_of(dstate_in, S, C);
        const Span places(offsets, 4, S + 1LL), scratch(workspace, 1, (long long)leet_attn_gated_scan_workspace_bytes(B, N, C, 1));
        for (const Span* o : {&to_x, &to_gate, &before, &scratch})
            if (shares_any(*o, {&rows_dh, &rows_gate, &rows_h, &rows_x, &in, &places})) return LEET_ERR_INVALID_ARG;
        if (shares_any(to_x, {&to_gate, &before, &behind, &scratch}) || shares_any(to_gate, {&before, &behind, &scratch}) ||
            shares_any(scratch, {&before, &behind}) || (dstate_in != dstate_out && overlap(before, behind)))
            return LEET_ERR_INVALID_ARG;
    }
    if (S == 0 || (N == 0 && (!dstate_in || dstate_in == dstate_out))) return LEET_OK;
    p.state_in = state_in;
    p.dstate_out = dstate_out;
    p.dstate_in = dstate_in;
    p.offsets = offsets;
    p.sequences = S;
    p.B = B; p.N = N; p.C = C;
    p.workspace = workspace;
    int dev = 0;
    status = leet::current_device(&dev);
    if (status != LEET_OK) return status;
    return done(leet::launch_gated_scan_backward(p, elem_of(dtype), elem_of(gate_dtype), mode, static_cast<hipStream_t>(stream)));
}

int leet_attn_gated_scan_step(const leet_attn_rows *x, const leet_attn_rows *gate, const leet_attn_rows *out,
                              float *state, int B, int C, int dtype, int gate_dtype, int mode, void *stream) {
    int status = scan_types_ok(dtype, gate_dtype, mode);
    if (status != LEET_OK) return status;
    if (B <= 0 || C <= 0 || !state || !aligned(state, 4)) return LEET_ERR_INVALID_ARG;
    if (C > 1 << 28) return LEET_ERR_TOO_LARGE;
    leet::GatedScanParams p = {};
    if (!rows_ok(x, B, 1, C, size_of(dtype), false) || !rows_ok(gate, B, 1, C, size_of(gate_dtype), false) ||
        !rows_ok(out, B, 1, C, size_of(dtype), true))
        return LEET_ERR_INVALID_ARG;
    // in place only element for element
    const Span rows_x = span_of(x, B, 1, C, (long long)size_of(dtype)), to = span_of(out, B, 1, C, (long long)size_of(dtype));
    const Span rows_gate = span_of(gate, B, 1, C, (long long)size_of(gate_dtype)), rows_state = states_of(state, B, C);
    if (!in_place_or_apart(to, rows_x) || !in_place_or_apart(to, rows_gate) ||
        shares_any(rows_state, {&rows_x, &rows_gate, &to}))
        return LEET_ERR_INVALID_ARG;
    p.vector = C % 4 == 0 && aligned(state, 16) && by_four(x, B, size_of(dtype)) && by_four(gate, B, size_of(gate_dtype)) &&
                       by_four(out, B, size_of(dtype)) ? 4 : 1;
    p.x = rows_in(x);
    p.gate = rows_in(gate);
    p.out = rows_out(out);
    p.state_out = state;
    p.B = B; p.C = C;
    int dev = 0;
    status = leet::current_device(&dev);
    if (status != LEET_OK) return status;
    return done(leet::launch_gated_step(p, elem_of(dtype), elem_of(gate_dtype), mode, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
