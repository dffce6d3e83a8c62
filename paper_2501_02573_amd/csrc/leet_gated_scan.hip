// The gated linear recurrence, element-wise in every channel:
//
//     h_t = a_t h_{t-1} + b_t              (a, b) = (z, x) | (exp z, x) | (sigmoid z, (1 - sigmoid z) x)
//
// and its backward pass.  With g_t = a_t D_t the gradient that flows on into h_{t-1},
//
//     D_t = dh_t + g_{t+1},   so   g_t = a_t g_{t+1} + a_t dh_t:
//
// the same recurrence from the last token to the first, with the same decays in the same places.
//
// A run of tokens is the map h -> A h + H with A the product of its decays and H what it leaves of a zero state; runs
// are joined by (A2, H2) after (A1, H1) = (A2 A1, A2 H1 + H2).  A wave takes kTokens tokens of 64 lanes' channels into
// registers and forms its run's (A, H); the waves of a workgroup lie behind one another in time and exchange their runs
// through LDS; each then knows the state before its first token and goes over its registers once more.  So inputs are
// read once and outputs written once, which is all that bounds it: a bf16 forward pass moves 6 bytes a token and channel
// for some ten operations.
//
// Packed sequences: where a sequence begins, the run so far is cut off.  That is decided by the offsets alone, so it
// is the same for all channels and no arithmetic carries anything over (zero times an infinity would).
#include "leet_gated_scan.hpp"
#include "leet_io.hpp"

namespace leet {

constexpr int kScanTokens = 16;  // of a wave at a time
constexpr int kScanWaves = 16;   // of a workgroup, at most

// The decay a and, for the moving average, 1 - a (as accurate as a itself however near 1 that is).
template <int kMode>
__device__ __forceinline__ void decay(float z, float& a, float& rest) {
    if constexpr (kMode == 0) a = z;
    else if constexpr (kMode == 1) a = expf(z);
    else {
        const float e = expf(-fabsf(z));
        const float large = 1.0f / (1.0f + e), small = e * large;
        a = z >= 0.0f ? large : small;
        rest = z >= 0.0f ? small : large;
    }
}

// Where the tokens t0 .. t0 + kScanTokens - 1 lie among packed sequences.  Lane i < kScanTokens looks at token t0 + i.
struct Places {
    int sequence;          // this lane's token's
    uint32_t first, last;  // tokens that begin, end a sequence
    uint32_t inside;       // tokens that belong to one

    Places() = default;
    __device__ __forceinline__ Places(const int* offsets, int sequences, int t0, int N, int lane) {
        const int t = t0 + min(lane, kScanTokens - 1);
        // the last sequence that begins at or before t: of empty ones at one place the one behind them
        int lo = 0, hi = sequences;  // offsets[lo] <= t < offsets[hi + 1], with offsets[S + 1] infinite
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (offsets[mid] <= t) lo = mid;
            else hi = mid - 1;
        }
        const bool in = lo < sequences && t < N && lane < kScanTokens;
        sequence = min(lo, sequences - 1);
        first = (uint32_t)__ballot(in && offsets[sequence] == t);
        last = (uint32_t)__ballot(in && offsets[sequence + 1] == t + 1);
        inside = (uint32_t)__ballot(in);
    }
    __device__ __forceinline__ int of(int i) const { return __builtin_amdgcn_readlane(sequence, i); }
};

template <int kElem, int kV>
__device__ __forceinline__ void load_channels(const RowsIn& r, int b, long long t, uint32_t c, float* f) {
    const char* row = r.data + (b * r.batch + t * r.token) * Io<kElem>::kBytes;
    Io<kElem>::template load<kV>(row + c * Io<kElem>::kBytes, f);
}
template <int kElem, int kV>
__device__ __forceinline__ void store_channels(const RowsOut& r, int b, long long t, uint32_t c, const float* f) {
    char* row = r.data + (b * r.batch + t * r.token) * Io<kElem>::kBytes;
    Io<kElem>::template store<kV>(row + c * Io<kElem>::kBytes, f);
}
template <int kV>
__device__ __forceinline__ void load_state(const float* s, int sequence, int C, uint32_t c, float* f) {
#pragma unroll
    for (int v = 0; v < kV; ++v) f[v] = s ? s[(size_t)sequence * C + c + v] : 0.0f;
}
template <int kV>
__device__ __forceinline__ void store_state(float* s, int sequence, int C, uint32_t c, const float* f) {
    if (!s) return;
#pragma unroll
    for (int v = 0; v < kV; ++v) s[(size_t)sequence * C + c + v] = f[v];
}

// Runs of the waves of a workgroup, two tiles' worth: a tile's are read while the next one's are written.
template <int kV>
struct Runs {
    float A[2][kScanWaves][64 * kV], H[2][kScanWaves][64 * kV];
    int cut[2][kScanWaves];  // a sequence begins (backward: ends) in the run: what came before it does not reach behind it
};

// Workgroup = one batch entry x 64 kV channels; its waves walk over the tokens in tiles of waves * kScanTokens.
template <int kX, int kG, int kMode, int kV, bool kPacked>
__global__ __launch_bounds__(64 * kScanWaves) void gated_scan_kernel(GatedScanParams p) {
    __shared__ Runs<kV> runs;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int b = (int)(blockIdx.x / (unsigned)p.columns), column = (int)(blockIdx.x % (unsigned)p.columns);
    const uint32_t c = (uint32_t)(column * 64 + lane) * kV;
    const bool live = c < (uint32_t)p.C;
    float carry[kV];
#pragma unroll
    for (int v = 0; v < kV; ++v) carry[v] = 0.0f;
    if (!kPacked && live) load_state<kV>(p.state_in, b, p.C, c, carry);

    int stage = 0;
    for (long long tile = 0; tile < p.N; tile += p.waves * kScanTokens, stage ^= 1) {
        const int t0 = (int)tile + wave * kScanTokens, count = min(max(p.N - t0, 0), kScanTokens);
        float a[kScanTokens][kV], h[kScanTokens][kV];
#pragma unroll
        for (int i = 0; i < kScanTokens; ++i) {
#pragma unroll
            for (int v = 0; v < kV; ++v) a[i][v] = h[i][v] = 0.0f;
            if (live && i < count) {
                load_channels<kG, kV>(p.gate, b, t0 + i, c, a[i]);
                load_channels<kX, kV>(p.x, b, t0 + i, c, h[i]);
            }
        }
        Places at = kPacked ? Places(p.offsets, p.sequences, t0, p.N, lane) : Places{};
        float A[kV], H[kV];
#pragma unroll
        for (int v = 0; v < kV; ++v) { A[v] = 1.0f; H[v] = 0.0f; }
#pragma unroll
        for (int i = 0; i < kScanTokens; ++i) {
            if (i >= count) continue;
            const bool first = kPacked && (at.first >> i & 1);
            float enters[kV];
            if (first && live) load_state<kV>(p.state_in, at.of(i), p.C, c, enters);
#pragma unroll
            for (int v = 0; v < kV; ++v) {
                float rest = 1.0f;
                decay<kMode>(a[i][v], a[i][v], rest);
                if (kMode == 2) h[i][v] *= rest;
                if (first) {
                    // the state is read here only: it may be overwritten as soon as this workgroup's runs are known
                    h[i][v] = fmaf(a[i][v], enters[v], h[i][v]);
                    H[v] = h[i][v];
                } else {
                    H[v] = fmaf(a[i][v], H[v], h[i][v]);
                    A[v] *= a[i][v];
                }
            }
        }
#pragma unroll
        for (int v = 0; v < kV; ++v) {
            runs.A[stage][wave][lane * kV + v] = A[v];
            runs.H[stage][wave][lane * kV + v] = H[v];
        }
        if (lane == 0) runs.cut[stage][wave] = kPacked && at.first != 0;
        __syncthreads();
        float before[kV];  // the state before this wave's first token
#pragma unroll
        for (int v = 0; v < kV; ++v) before[v] = carry[v];
        for (int w = 0; w < p.waves; ++w) {
            const bool cut = kPacked && runs.cut[stage][w];
#pragma unroll
            for (int v = 0; v < kV; ++v) {
                const float Hw = runs.H[stage][w][lane * kV + v];
                if (w == wave) before[v] = carry[v];
                carry[v] = cut ? Hw : fmaf(runs.A[stage][w][lane * kV + v], carry[v], Hw);
            }
        }
#pragma unroll
        for (int i = 0; i < kScanTokens; ++i) {
            if (i >= count) continue;
            const bool first = kPacked && (at.first >> i & 1);
#pragma unroll
            for (int v = 0; v < kV; ++v) {
                before[v] = first ? h[i][v] : fmaf(a[i][v], before[v], h[i][v]);
                h[i][v] = before[v];
            }
            if (live && (!kPacked || (at.inside >> i & 1))) {
                store_channels<kX, kV>(p.out, b, t0 + i, c, h[i]);
                if (kPacked && (at.last >> i & 1)) store_state<kV>(p.state_out, at.of(i), p.C, c, h[i]);
            }
        }
    }
    if (!kPacked && live && wave == 0) store_state<kV>(p.state_out, b, p.C, c, carry);
    if (kPacked && p.state_out && live)
        for (int s = wave; s < p.sequences; s += p.waves)
            if (p.offsets[s] == p.offsets[s + 1]) {
                float f[kV];
                load_state<kV>(p.state_in, s, p.C, c, f);
                store_state<kV>(p.state_out, s, p.C, c, f);
            }
}

// The same from the last tile to the first.  The run of a wave maps the gradient that comes in from behind its last
// token to the one that goes out before its first.
template <int kX, int kG, int kMode, int kV, bool kPacked>
__global__ __launch_bounds__(64 * kScanWaves) void gated_scan_backward_kernel(GatedScanParams p) {
    __shared__ Runs<kV> runs;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int b = (int)(blockIdx.x / (unsigned)p.columns), column = (int)(blockIdx.x % (unsigned)p.columns);
    const uint32_t c = (uint32_t)(column * 64 + lane) * kV;
    const bool live = c < (uint32_t)p.C;
    float carry[kV];
#pragma unroll
    for (int v = 0; v < kV; ++v) carry[v] = 0.0f;
    if (!kPacked && live) load_state<kV>(p.dstate_out, b, p.C, c, carry);

    const int tokens = p.waves * kScanTokens;
    int stage = 0;
    for (long long tile = ((long long)p.N - 1) / tokens * tokens; tile >= 0; tile -= tokens, stage ^= 1) {
        const int t0 = (int)tile + wave * kScanTokens, count = min(max(p.N - t0, 0), kScanTokens);
        float a[kScanTokens][kV], d[kScanTokens][kV], rest[kScanTokens][kV];
#pragma unroll
        for (int i = 0; i < kScanTokens; ++i) {
#pragma unroll
            for (int v = 0; v < kV; ++v) a[i][v] = d[i][v] = rest[i][v] = 0.0f;
            if (live && i < count) {
                load_channels<kG, kV>(p.gate, b, t0 + i, c, a[i]);
                load_channels<kX, kV>(p.dh, b, t0 + i, c, d[i]);
            }
        }
        Places at = kPacked ? Places(p.offsets, p.sequences, t0, p.N, lane) : Places{};
        float A[kV], G[kV];
#pragma unroll
        for (int v = 0; v < kV; ++v) { A[v] = 1.0f; G[v] = 0.0f; }
#pragma unroll
        for (int i = kScanTokens - 1; i >= 0; --i) {
            if (i >= count) continue;
            const bool last = kPacked && (at.last >> i & 1);
            float leaves[kV];
            if (last && live) load_state<kV>(p.dstate_out, at.of(i), p.C, c, leaves);
#pragma unroll
            for (int v = 0; v < kV; ++v) {
                decay<kMode>(a[i][v], a[i][v], rest[i][v]);
                if (last) {
                    d[i][v] += leaves[v];
                    G[v] = a[i][v] * d[i][v];
                } else {
                    G[v] = a[i][v] * (d[i][v] + G[v]);
                    A[v] *= a[i][v];
                }
            }
        }
#pragma unroll
        for (int v = 0; v < kV; ++v) {
            runs.A[stage][wave][lane * kV + v] = A[v];
            runs.H[stage][wave][lane * kV + v] = G[v];
        }
        if (lane == 0) runs.cut[stage][wave] = kPacked && at.last != 0;
        __syncthreads();
        float behind[kV];  // the gradient that comes in from behind this wave's last token
#pragma unroll
        for (int v = 0; v < kV; ++v) behind[v] = carry[v];
        for (int w = p.waves - 1; w >= 0; --w) {
            const bool cut = kPacked && runs.cut[stage][w];
#pragma unroll
            for (int v = 0; v < kV; ++v) {
                const float Gw = runs.H[stage][w][lane * kV + v];
                if (w == wave) behind[v] = carry[v];
                carry[v] = cut ? Gw : fmaf(runs.A[stage][w][lane * kV + v], carry[v], Gw);
            }
        }
#pragma unroll
        for (int i = kScanTokens - 1; i >= 0; --i) {
            if (i >= count || !live || (kPacked && !(at.inside >> i & 1))) continue;
            const bool last = kPacked && (at.last >> i & 1), first = kPacked ? (at.first >> i & 1) : t0 + i == 0;
            float before[kV], x[kV], dx[kV], dgate[kV];
            if (first) load_state<kV>(p.state_in, kPacked ? at.of(i) : b, p.C, c, before);
            else load_channels<kX, kV>(p.h, b, t0 + i - 1, c, before);
            if (kMode == 2) load_channels<kX, kV>(p.x, b, t0 + i, c, x);
#pragma unroll
            for (int v = 0; v < kV; ++v) {
                const float D = last ? d[i][v] : d[i][v] + behind[v];
                behind[v] = a[i][v] * D;
                if (kMode == 0) { dgate[v] = D * before[v]; dx[v] = D; }
                else if (kMode == 1) { dgate[v] = behind[v] * before[v]; dx[v] = D; }
                else { dgate[v] = behind[v] * rest[i][v] * (before[v] - x[v]); dx[v] = D * rest[i][v]; }
            }
            store_channels<kX, kV>(p.dx, b, t0 + i, c, dx);
            store_channels<kG, kV>(p.dgate, b, t0 + i, c, dgate);
            if (kPacked && first) store_state<kV>(p.dstate_in, at.of(i), p.C, c, behind);
        }
    }
    if (!kPacked && live && wave == 0) store_state<kV>(p.dstate_in, b, p.C, c, carry);
    if (kPacked && p.dstate_in && live)
        for (int s = wave; s < p.sequences; s += p.waves)
            if (p.offsets[s] == p.offsets[s + 1]) {
                float f[kV];
                load_state<kV>(p.dstate_out, s, p.C, c, f);
                store_state<kV>(p.dstate_in, s, p.C, c, f);
            }
}

// One token of every sequence: state <- a state + b, out = state.  One thread per kV channels.
template <int kX, int kG, int kMode, int kV>
__global__ __launch_bounds__(256) void gated_step_kernel(GatedScanParams p) {
    const uint32_t c = (blockIdx.x * 256 + threadIdx.x) * kV;
    if (c >= (uint32_t)p.C) return;
    for (int b = blockIdx.y; b < p.B; b += gridDim.y) {
        float a[kV], x[kV], s[kV];
        load_channels<kG, kV>(p.gate, b, 0, c, a);
        load_channels<kX, kV>(p.x, b, 0, c, x);
        char* state = reinterpret_cast<char*>(p.state_out + (size_t)b * p.C + c);
        Io<0>::load<kV>(state, s);
#pragma unroll
        for (int v = 0; v < kV; ++v) {
            float rest = 1.0f;
            decay<kMode>(a[v], a[v], rest);
            s[v] = fmaf(a[v], s[v], kMode == 2 ? rest * x[v] : x[v]);
        }
        Io<0>::store<kV>(state, s);
        store_channels<kX, kV>(p.out, b, 0, c, s);
    }
}

// which: 0 forward, 1 backward
template <int kX, int kG, int kMode, int kV>
static void launch_scan_v(const GatedScanParams& p, int which, hipStream_t stream) {
    const dim3 grid((unsigned)p.B * (unsigned)p.columns), block(64 * (unsigned)p.waves);
    if (which == 0) {
        if (p.offsets) hipLaunchKernelGGL((gated_scan_kernel<kX, kG, kMode, kV, true>), grid, block, 0, stream, p);
        else hipLaunchKernelGGL((gated_scan_kernel<kX, kG, kMode, kV, false>), grid, block, 0, stream, p);
    } else {
        if (p.offsets) hipLaunchKernelGGL((gated_scan_backward_kernel<kX, kG, kMode, kV, true>), grid, block, 0, stream, p);
        else hipLaunchKernelGGL((gated_scan_backward_kernel<kX, kG, kMode, kV, false>), grid, block, 0, stream, p);
    }
}

template <int kX, int kG, int kMode>
static void launch_scan_m(const GatedScanParams& p, int which, hipStream_t stream) {
    if (which == 2) {
        const int v = p.vector >= 4 ? 4 : 1;
        const unsigned blocks = (unsigned)((p.C / v + (p.C % v != 0) + 255) / 256);
        const dim3 grid(blocks, (unsigned)(p.B < 65535 ? p.B : 65535)), block(256);
        if (v >= 4) hipLaunchKernelGGL((gated_step_kernel<kX, kG, kMode, 4>), grid, block, 0, stream, p);
        else hipLaunchKernelGGL((gated_step_kernel<kX, kG, kMode, 1>), grid, block, 0, stream, p);
    } else if (p.vector >= 2) launch_scan_v<kX, kG, kMode, 2>(p, which, stream);
    else launch_scan_v<kX, kG, kMode, 1>(p, which, stream);
}

template <int kX, int kG>
static hipError_t launch_scan_g(const GatedScanParams& p, int mode, int which, hipStream_t stream) {
    if (mode == 0) launch_scan_m<kX, kG, 0>(p, which, stream);
    else if (mode == 1) launch_scan_m<kX, kG, 1>(p, which, stream);
    else launch_scan_m<kX, kG, 2>(p, which, stream);
    return hipGetLastError();
}

static hipError_t launch_scan(const GatedScanParams& p, int elem, int gate_elem, int mode, int which, hipStream_t stream) {
    if (elem == 0) return launch_scan_g<0, 0>(p, mode, which, stream);
    if (elem == 1) return gate_elem ? launch_scan_g<1, 1>(p, mode, which, stream) : launch_scan_g<1, 0>(p, mode, which, stream);
    return gate_elem ? launch_scan_g<2, 2>(p, mode, which, stream) : launch_scan_g<2, 0>(p, mode, which, stream);
}

static void plan_scan(GatedScanParams* p) {
    const int v = p->vector >= 2 ? 2 : 1;
    p->columns = (p->C + 64 * v - 1) / (64 * v);
    const int need = (p->N + kScanTokens - 1) / kScanTokens;
    p->waves = need < 1 ? 1 : need < kScanWaves ? need : kScanWaves;  // no tokens: one that hands the states on
}

hipError_t launch_gated_scan(GatedScanParams p, int elem, int gate_elem, int mode, hipStream_t stream) {
    plan_scan(&p);
    return launch_scan(p, elem, gate_elem, mode, 0, stream);
}

hipError_t launch_gated_scan_backward(GatedScanParams p, int elem, int gate_elem, int mode, hipStream_t stream) {
    plan_scan(&p);
    return launch_scan(p, elem, gate_elem, mode, 1, stream);
}

hipError_t launch_gated_step(GatedScanParams p, int elem, int gate_elem, int mode, hipStream_t stream) {
    return launch_scan(p, elem, gate_elem, mode, 2, stream);
}

}  // namespace leet
