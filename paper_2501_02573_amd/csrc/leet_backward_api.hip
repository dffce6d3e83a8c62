// C ABI of the attention's backward pass: argument checks, segments, launches.  Nothing here touches tensor data.
#include <math.h>

#include "../../include/leet_attn.h"
#include "leet_backward.hpp"
#include "leet_common.hpp"
#include "leet_host.hpp"
#include "leet_overlap.hpp"

namespace leet {
hipError_t launch_state_pass(const float* state_in, float* state_out, int BH, int D, int DV, hipStream_t stream);
hipError_t launch_seg_scan(float* seg_state, const float* state_in, float* state_copy, const float* gamma, int BH, int H,
                           int nseg, int seg_tokens, int step, int D, int DV, hipStream_t stream);
}  // namespace leet

namespace {

using leet::kChunk;
using leet::Span;

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

bool shape_ok(int r, int dv, int dtype) {
    if (dtype != LEET_F32 && dtype != LEET_BF16 && dtype != LEET_F16) return false;
    return (r == dv && (r == 64 || r == 128)) || (r == 128 && dv == 256 && dtype != LEET_F32);
}

struct Plan {
    int nseg, seg_chunks;
    bool tiles;       // the kernel that takes a compute unit a sequence
    size_t ws_bytes;  // states of both directions at the boundaries of segments
};

// What a call takes, in microseconds, by its number of segments.  Workgroups go to the eight XCDs in turn, and an XCD holds
// `resident` of them on 32 compute units: a chunk takes them alone_us while each has a unit to itself, full_us when all are there.
// A call is its walk and, with segments, the pre-pass over the states and the scan, each the smooth maximum
// (x^p + y^p)^(1/p) of that and of its memory traffic.  Fitted (3 to 8 % rms) to runs of BH 1..512, N 64..32768 and 1 to 64
// segments; the picks are 0.4 % (16-bit, 128), 1.2 % (16-bit, 64) and 0.7 % (fp32) slower than the best of each run on average.  16-bit
// is bf16; fp16, 6 to 18 % slower, has the same picks, 0.8 % (128) and 2.9 % (64) off the best of 15 shapes (BH 128 N 4096, 64: 222 us,
// 180 with two segments; bf16 192 and 170).  Width 256 by fewer runs (BH 32 N 2048, 1 to 8 segments: 291 221 168 140 178 153 us).
struct CostModel {
    double call_us, segments_us, segment_us;  // fixed: of a call, of having segments, of each of them
    double alone_us, full_us, round_us;       // walk: a chunk; what a round of workgroups begins with
    double state_alone_us, state_full_us;     // pre-pass: a chunk
    double bytes_per_us, p;
    int resident;
};
constexpr CostModel kModel16x128 = {3.0, 7.9, 0.32, 2.41, 3.82, 9.0, 1.94, 3.08, 4.70e6, 4.0, 64};
constexpr CostModel kModel16x64 = {7.3, 5.3, 0.323, 2.13, 3.33, 0.1, 1.09, 1.15, 5.39e6, 4.0, 128};
constexpr CostModel kModel16x256 = {3.0, 9.7, 0.335, 9.0, 22.0, 8.0, 4.0, 8.0, 4.50e6, 20.0, 64};
constexpr CostModel kModel32x128 = {3.0, 7.6, 0.377, 11.8, 25.5, 8.7, 5.42, 12.5, 3.50e6, 20.0, 64};
constexpr CostModel kModel32x64 = {3.0, 6.0, 0.337, 4.85, 8.10, 3.4, 1.99, 2.60, 4.28e6, 20.0, 64};

double smooth_max(double a, double b, double p) { return pow(pow(a, p) + pow(b, p), 1.0 / p); }

double predicted_us(const CostModel& m, long BH, int N, int r, int dv, int size, int nseg, int seg_chunks) {
    auto chunk_us = [&](long units, double alone, double full) {  // of all rounds of an XCD's workgroups
        const long rest = units % m.resident;
        return units / m.resident * full + (rest == 0 ? 0.0 : rest <= 32 ? alone : m.resident == 64 ? full
                                                 : alone + (full - alone) * (rest - 32) / (m.resident - 32));
    };
    const int roles = r == dv ? 3 : 2;  // width 256: dv has a launch of its own, counted in alone_us
    const long units = roles * ((BH * nseg + 7) / 8);
    // walks read seven tensors' worth (dk's and dv's common ones meet in the cache) and write three
    const double tensor = (double)BH * N * (r + dv) / 2 * size;
    double us = m.call_us + smooth_max(seg_chunks * chunk_us(units, m.alone_us, m.full_us) +
                                           m.round_us * ((units + m.resident - 1) / m.resident),
                                       10 * tensor / m.bytes_per_us, m.p);
    if (nseg > 1)
        us += m.segments_us + m.segment_us * nseg +
              smooth_max(seg_chunks * chunk_us(2 * ((BH * (nseg - 1) + 7) / 8), m.state_alone_us, m.state_full_us),
                         4 * tensor * (nseg - 1) / nseg / m.bytes_per_us, m.p);
    return us;
}

bool make_plan(long BH, int N, int r, int dv, int dtype, int segments, Plan* plan) {
    const int nchunks = (N + kChunk - 1) / kChunk, size = dtype == LEET_F32 ? 4 : 2;
    const CostModel& m = dtype == LEET_F32 ? (r == 64 ? kModel32x64 : kModel32x128)
                                           : dv == 256 ? kModel16x256 : r == 64 ? kModel16x64 : kModel16x128;
    double best = 0.0;
    auto consider = [&](int want) {  // a later candidate has to be 2 % better
        const int seg_chunks = (nchunks + want - 1) / want, nseg = (nchunks + seg_chunks - 1) / seg_chunks;
        const double us = predicted_us(m, BH, N, r, dv, size, nseg, seg_chunks);
        if (best > 0.0 && us >= best * 0.98) return;
        best = us;
        plan->nseg = nseg;
        plan->seg_chunks = seg_chunks;
    };
    if (segments > 0) consider(segments < nchunks ? segments : nchunks);
    else
        // 16-bit segments have two chunks at least
        for (int want : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64})
            if (want == 1 || (dtype == LEET_F32 ? want <= nchunks : 2 * want <= nchunks)) consider(want);
    // The kernel that takes a compute unit a sequence: no more workgroups than an XCD has compute units.  A
    // chunk takes it 2.3 us in a few workgroups, 2.7 in 192.  us, here against the best of the other: BH 4 N 512 24 26, N 1024 43
    // 30; BH 32 N 1024 43 46, N 2048 83 68; BH 64 N 4096 177 200, N 16384 715 740; BH 85 N 4096 (a second round) 302 270.
    // (Sequences of one or two chunks go to the other, which takes their scores and states in two terms.)
    plan->tiles = r == 128 && dv == 128 && dtype != LEET_F32 && nchunks > 2 && 3 * ((BH + 7) / 8) <= 32 &&
                  (segments == 0 ? nchunks * (2.3 + 0.0065 * BH) + 5.0 < best : plan->nseg == 1);
    if (plan->tiles) {
        plan->nseg = 1;
        plan->seg_chunks = nchunks;
    }
    plan->ws_bytes = (size_t)2 * BH * (plan->nseg - 1) * r * dv * sizeof(float);
    // fewer than 2^32 threads a launch: workgroups of up to 512 threads, three a segment; the scan, a thread for four elements of the
    // states of both directions
    return BH * plan->nseg < 1L << 21 && (plan->nseg == 1 || 2 * BH * (r * dv / 4) < 1L << 32);
}

// make_plan with the last plan of the calling thread kept: a call asks for it twice, and a program's calls mostly repeat one shape.
bool call_plan(long BH, int N, int r, int dv, int dtype, int segments, Plan* plan) {
    struct Kept {
        long BH = 0;  // 0: nothing kept
        int N, r, dv, dtype, segments;
        Plan plan;
    };
    static thread_local Kept kept;
    if (kept.BH != BH || kept.N != N || kept.r != r || kept.dv != dv || kept.dtype != dtype || kept.segments != segments) {
        kept.BH = 0;
        if (!make_plan(BH, N, r, dv, dtype, segments, &kept.plan)) return false;
        kept.BH = BH; kept.N = N; kept.r = r; kept.dv = dv;
        kept.dtype = dtype; kept.segments = segments;
    }
    *plan = kept.plan;
    return true;
}

}  // namespace

extern "C" {

size_t leet_attn_backward_workspace_bytes(int B, int H, int N, int r, int dv, int dtype, int segments) {
    Plan plan;
    if (B <= 0 || H <= 0 || N <= 0 || segments < 0 || !shape_ok(r, dv, dtype) || (long)B * H >= 1L << 21 || N > 1 << 30 ||
        !call_plan((long)B * H, N, r, dv, dtype, segments, &plan))
        return 0;
    return plan.ws_bytes;
}

int leet_attn_backward(const void *dout, const void *q, const void *k, const void *v, const float *gamma,
                       void *dq, void *dk, void *dv_out, const float *state_in, const float *dstate_out, float *dstate_in,
                       void *workspace, size_t workspace_bytes, int segments,
                       int B, int H, int N, int r, int dv, int dtype, int mask, void *stream) {
    if (mask != LEET_MASK_DECAY && mask != LEET_MASK_CAUSAL) return LEET_ERR_INVALID_ARG;
    if (B <= 0 || H <= 0 || N < 0 || r <= 0 || dv <= 0 || segments < 0) return LEET_ERR_INVALID_ARG;
    if (mask == LEET_MASK_CAUSAL) gamma = nullptr;
    if ((N > 0 && (!dout || !q || !k || !v || !dq || !dk || !dv_out)) || (!gamma && mask == LEET_MASK_DECAY))
        return LEET_ERR_INVALID_ARG;
    if (!shape_ok(r, dv, dtype)) return LEET_ERR_UNSUPPORTED;
    for (const void* t : {dout, q, k, v, (const void*)dq, (const void*)dk, (const void*)dv_out, (const void*)state_in,
                          (const void*)dstate_out, (const void*)dstate_in})
        if (!aligned16(t)) return LEET_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(gamma) & 3u) || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return LEET_ERR_INVALID_ARG;
    const long BH = (long)B * H;
    if (BH >= 1L << 21 || N > 1 << 30) return LEET_ERR_TOO_LARGE;
    Plan plan = {1, 0, false, 0};
    if (N > 0 && !call_plan(BH, N, r, dv, dtype, segments, &plan)) return LEET_ERR_TOO_LARGE;
    if (plan.ws_bytes && (!workspace || workspace_bytes < plan.ws_bytes)) return LEET_ERR_INVALID_ARG;

    const long long isz = dtype == LEET_F32 ? 4 : 2, rows = (long long)BH * N, states = (long long)BH * r * dv;
    const Span outs[] = {Span(dq, isz, rows * r), Span(dk, isz, rows * r), Span(dv_out, isz, rows * dv), Span(dstate_in, 4, states),
                         Span(plan.ws_bytes ? workspace : nullptr, 1, (long long)plan.ws_bytes)};
    const Span ins[] = {Span(dout, isz, rows * dv), Span(q, isz, rows * r), Span(k, isz, rows * r), Span(v, isz, rows * dv),
                        Span(gamma, 4, H), Span(state_in, 4, states), Span(dstate_out, 4, states)};
    for (const Span& out : outs) {
        for (const Span& in : ins)
            if (overlap(out, in)) return LEET_ERR_INVALID_ARG;
        for (const Span& other : outs)
            if (&other != &out && overlap(out, other)) return LEET_ERR_INVALID_ARG;
    }

    int dev = 0;
    const int status = leet::current_device(&dev);
    if (status != LEET_OK) return status;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (N == 0) {
        // the state is handed on as it is, and so is its gradient
        const hipError_t e = leet::launch_state_pass(dstate_out, dstate_in, (int)BH, r, dv, s);
        return e == hipSuccess ? LEET_OK : LEET_ERR_LAUNCH;
    }

    float* slots = static_cast<float*>(workspace);
    float* slots_back = slots + plan.ws_bytes / 2 / sizeof(float);
    leet::BwdParams p = {};
    p.gamma = gamma;
    p.BH = (int)BH; p.H = H; p.N = N;
    p.nseg = plan.nseg; p.seg_chunks = plan.seg_chunks;
    // dq: the state transposed, [dv][r], in the order of the tokens; dk: the gradient of the state transposed, reversed; dv:
    // that gradient, [r][dv].  Slots hold [dv][r].
    const leet::BwdRole of_q = {dout, v, k, dq, state_in, nullptr, slots, 1, dv, r, 1, 0};
    const leet::BwdRole of_k = {v, dout, q, dk, dstate_out, nullptr, slots_back, 1, dv, r, 1, 1};
    const leet::BwdRole of_v = {k, q, dout, dv_out, dstate_out, dstate_in, slots_back, dv, 1, 1, r, 1};

    const bool f32 = dtype == LEET_F32, f16 = dtype == LEET_F16, fine = dstate_in != nullptr;
    hipError_t e = hipSuccess;
    p.role[0] = of_q;
    p.role[1] = of_k;
    p.roles = 2;
    if (plan.nseg > 1) {
        e = f32 ? leet::launch_bwd_f32_states(p, r, s) : leet::launch_bwd_16bit_states(p, dv, r, f16, fine, s);
        if (e == hipSuccess)
            e = leet::launch_seg_scan(slots, nullptr, nullptr, gamma, 2 * (int)BH, H, plan.nseg, plan.seg_chunks * kChunk, 1, dv, r, s);
    }
    if (e == hipSuccess && r == dv) {
        p.role[2] = of_v;
        p.roles = 3;
        e = f32 ? leet::launch_bwd_f32_walk(p, r, s)
            : plan.tiles ? leet::launch_bwd_16bit_tiles(p, f16, fine, s)
                         : leet::launch_bwd_16bit_walk(p, r, r, f16, fine, s);
    } else if (e == hipSuccess) {
        e = leet::launch_bwd_16bit_walk(p, dv, r, f16, fine, s);
        p.role[0] = of_v;
        p.roles = 1;
        if (e == hipSuccess) e = leet::launch_bwd_16bit_walk(p, r, dv, f16, fine, s);
    }
    return e == hipSuccess ? LEET_OK : LEET_ERR_LAUNCH;
}

}  // extern "C"
