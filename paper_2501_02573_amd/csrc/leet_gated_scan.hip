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

#ifndef SCAN_TOKENS
#define SCAN_TOKENS 8
#define SCAN_WAVES 16
#endif
constexpr int kScanTokens = SCAN_TOKENS;  // of a wave at a time
constexpr int kScanWaves = SCAN_WAVES;   // of a workgroup, at most

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

// Channel c of token t: a uniform address plus a lane's 32-bit offset.
template <int kElem>
__device__ __forceinline__ const char* row_at(const RowsIn& r, int b, long long t, uint32_t c) {
    return r.data + (b * r.batch + t * r.token) * Io<kElem>::kBytes + c * Io<kElem>::kBytes;
}
template <int kElem, int kV>
__device__ __forceinline__ void load_channels(const RowsIn& r, int b, long long t, uint32_t c, float* f) {
    Io<kElem>::template load<kV>(row_at<kElem>(r, b, t, c), f);
}
template <int kV>
__device__ __forceinline__ void zero(float* f) {
#pragma unroll
    for (int v = 0; v < kV; ++v) f[v] = 0.0f;
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

// What the tiles of a column block tell one another.  A tile's run (A, H) is known as soon as its inputs are; the state
// behind it (its inclusive state) when the state before it is.  Each is published by stores of eight bytes that no fence
// has to order: a word that has not been written holds kUnset, which no value is published as.
constexpr uint32_t kUnset = 0xffffffffu;  // a NaN that arithmetic does not produce; published as another one

__device__ __forceinline__ uint32_t publishable(float f) {
    const uint32_t u = __builtin_bit_cast(uint32_t, f);
    return u == kUnset ? 0x7fc00000u : u;
}
__device__ __forceinline__ void publish(uint64_t* at, float lo, float hi) {
    __hip_atomic_store(at, (uint64_t)publishable(hi) << 32 | publishable(lo), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint64_t look(const uint64_t* at) {
    return __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float low(uint64_t w) { return __builtin_bit_cast(float, (uint32_t)w); }
__device__ __forceinline__ float high(uint64_t w) { return __builtin_bit_cast(float, (uint32_t)(w >> 32)); }
__device__ __forceinline__ bool is_set(uint64_t w) { return (uint32_t)w != kUnset && (uint32_t)(w >> 32) != kUnset; }

// Workspace: a line for the ticket counter, then of every tile the runs of its channels (A, H: eight bytes a channel),
// then of every tile the inclusive states of its channels, four bytes a channel in pairs (a lone channel: twice itself).
struct Board {
    uint64_t *runs, *states;
    long long tile;  // words of a tile's runs
    static constexpr size_t kHeader = 256;

    template <int kV>
    __device__ __forceinline__ static Board of(const GatedScanParams& p, int block, int lane) {
        const long long blocks = (long long)p.B * p.columns, channels = blocks * 64 * kV;
        uint64_t* words = reinterpret_cast<uint64_t*>(static_cast<char*>(p.workspace) + kHeader);
        Board b;
        b.runs = words + ((long long)block * 64 + lane) * kV;
        b.states = words + channels * p.tiles + (long long)block * 64 + lane;
        b.tile = channels;
        return b;
    }
    template <int kV>
    __device__ __forceinline__ void publish_run(int k, const float* A, const float* H) const {
#pragma unroll
        for (int v = 0; v < kV; ++v) publish(runs + k * tile + v, A[v], H[v]);
    }
    template <int kV>
    __device__ __forceinline__ void publish_state(int k, const float* s) const {
        publish(states + k * (tile / kV), s[0], s[kV - 1]);
    }

    // The state behind tile k of the chain: looks back over what has been published until it meets an inclusive state,
    // kWindow tiles at a time, and waits for those that have published nothing.  Every wait ends: a tile publishes its
    // run (or its state) without waiting for anything, and tiles are taken in the order of the chain, so all that are
    // waited for belong to workgroups that are running already.
    template <int kV>
    __device__ __forceinline__ void state_behind(int k, bool live, float* state) const {
        constexpr int kWindow = 4;
        float A[kV], H[kV];
#pragma unroll
        for (int v = 0; v < kV; ++v) { A[v] = 1.0f; H[v] = 0.0f; }
        while (true) {
            uint64_t run[kWindow][kV], whole[kWindow];
#pragma unroll
            for (int u = 0; u < kWindow; ++u) {
                const int j = k - u < 0 ? 0 : k - u;
                whole[u] = live ? look(states + j * (tile / kV)) : 0;
#pragma unroll
                for (int v = 0; v < kV; ++v) run[u][v] = live ? look(runs + j * tile + v) : 0;
            }
            int seen = 0;
#pragma unroll
            for (int u = 0; u < kWindow; ++u) {
                if (seen != u || u > k) continue;  // behind one that has to be waited for, or before the first tile
                if (__all(is_set(whole[u]))) {
#pragma unroll
                    for (int v = 0; v < kV; ++v) state[v] = fmaf(A[v], v ? high(whole[u]) : low(whole[u]), H[v]);
                    return;
                }
                bool set = true;
#pragma unroll
                for (int v = 0; v < kV; ++v) set = set && is_set(run[u][v]);
                if (!__all(set)) continue;
#pragma unroll
                for (int v = 0; v < kV; ++v) {
                    H[v] = fmaf(A[v], high(run[u][v]), H[v]);
                    A[v] *= low(run[u][v]);
                }
                ++seen;
            }
            k -= seen;
        }
    }
};

// The workspace before a launch: no ticket taken, nothing published.
__global__ __launch_bounds__(256) void gated_scan_clear_kernel(u32x4* words, size_t count) {
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i < count) words[i] = i < Board::kHeader / 16 ? u32x4{0, 0, 0, 0} : u32x4{kUnset, kUnset, kUnset, kUnset};
}

// Shared by the waves of a workgroup.
template <int kV>
struct Shared {
    float A[kScanWaves][64 * kV], H[kScanWaves][64 * kV];  // the waves' runs
    int cut[kScanWaves];  // a sequence begins (backward: ends) in the run: what came before it does not reach behind it
    float carry[64 * kV];
    unsigned ticket;
};

// The tile of a workgroup: column block `block` of all batch entries, tile k of its chain.
template <int kV>
__device__ __forceinline__ void take_tile(const GatedScanParams& p, Shared<kV>& shared, int* block, int* k) {
    unsigned ticket = blockIdx.x;
    const unsigned blocks = (unsigned)p.B * (unsigned)p.columns;
    if (p.tiles > 1) {
        // in the order in which workgroups start, whatever that is
        if (threadIdx.x == 0) shared.ticket = atomicAdd(static_cast<unsigned*>(p.workspace), 1u);
        __syncthreads();
        ticket = (unsigned)__builtin_amdgcn_readfirstlane((int)shared.ticket);
    }
    *block = (int)(ticket % blocks);
    *k = (int)(ticket / blocks);
}

// Joins the runs of a tile's waves in the order of the chain (kBackward: from the last wave to the first).  before[] is
// the state before this wave's run, after the state behind the whole tile (wave 0 only).  entering: wave 0's, the state
// before the whole tile where the chain begins.
template <int kV, bool kBackward, bool kPacked>
__device__ __forceinline__ void join_runs(const GatedScanParams& p, Shared<kV>& shared, int block, int k, int wave, int lane,
                                          bool live, const float* A, const float* H, bool cut, const float* entering,
                                          float* before, float* after) {
#pragma unroll
    for (int v = 0; v < kV; ++v) {
        shared.A[wave][lane * kV + v] = A[v];
        shared.H[wave][lane * kV + v] = H[v];
    }
    if (kPacked && lane == 0) shared.cut[wave] = cut;
    __syncthreads();
    float mineA[kV], mineH[kV], allA[kV], allH[kV];
    bool mine_cut = false, all_cut = false;
#pragma unroll
    for (int v = 0; v < kV; ++v) {
        allA[v] = mineA[v] = 1.0f;
        allH[v] = mineH[v] = 0.0f;
    }
    const int ahead = kBackward ? p.waves - 1 - wave : wave;  // runs that come before this wave's
    const int last = wave == 0 ? p.waves : ahead;             // wave 0 goes on to the end: it joins the tile to the others
    for (int i = 0; i < last; ++i) {
        const int w = kBackward ? p.waves - 1 - i : i;
        if (i == ahead) {
            mine_cut = all_cut;
#pragma unroll
            for (int v = 0; v < kV; ++v) { mineA[v] = allA[v]; mineH[v] = allH[v]; }
        }
        const bool here = kPacked && shared.cut[w];
        all_cut = all_cut || here;
#pragma unroll
        for (int v = 0; v < kV; ++v) {
            const float Hw = shared.H[w][lane * kV + v], Aw = shared.A[w][lane * kV + v];
            allH[v] = here ? Hw : fmaf(Aw, allH[v], Hw);
            allA[v] *= Aw;
        }
    }
    if (wave != 0) {
        mine_cut = all_cut;
#pragma unroll
        for (int v = 0; v < kV; ++v) { mineA[v] = allA[v]; mineH[v] = allH[v]; }
    } else {
        float carry[kV];
        const Board board = Board::of<kV>(p, block, lane);
        if (k == 0) {
#pragma unroll
            for (int v = 0; v < kV; ++v) carry[v] = entering[v];
        } else {
            if (live && !all_cut) board.publish_run<kV>(k, allA, allH);
            if (live && all_cut) board.publish_state<kV>(k, allH);
            board.state_behind<kV>(k - 1, live, carry);
        }
#pragma unroll
        for (int v = 0; v < kV; ++v) {
            after[v] = all_cut ? allH[v] : fmaf(allA[v], carry[v], allH[v]);
            shared.carry[lane * kV + v] = carry[v];
        }
        if (live && p.tiles > 1 && (k == 0 || !all_cut)) board.publish_state<kV>(k, after);
    }
    __syncthreads();
#pragma unroll
    for (int v = 0; v < kV; ++v) before[v] = mine_cut ? mineH[v] : fmaf(mineA[v], shared.carry[lane * kV + v], mineH[v]);
}

// States of empty packed sequences are handed on; the sequences are spread over the tiles and waves.
template <int kV>
__device__ __forceinline__ void pass_on(const GatedScanParams& p, const float* from, float* to, int k, int wave, uint32_t c) {
    if (!to) return;
    for (int s = k * p.waves + wave; s < p.sequences; s += p.tiles * p.waves)
        if (p.offsets[s] == p.offsets[s + 1]) {
            float f[kV];
            load_state<kV>(from, s, p.C, c, f);
            store_state<kV>(to, s, p.C, c, f);
        }
}

// Workgroup = one tile of waves * kScanTokens tokens x 64 kV channels of one batch entry.
template <int kX, int kG, int kMode, int kV, bool kPacked>
__global__ __launch_bounds__(64 * kScanWaves) void gated_scan_kernel(GatedScanParams p) {
    __shared__ Shared<kV> shared;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int block, k;
    take_tile<kV>(p, shared, &block, &k);
    const int b = block / p.columns;
    const uint32_t c = (uint32_t)((block - b * p.columns) * 64 + lane) * kV;
    const bool live = c < (uint32_t)p.C;
    const int t0 = (k * p.waves + wave) * kScanTokens, count = min(max(p.N - t0, 0), kScanTokens);

    typename Io<kG>::template Raw<kV> z[kScanTokens];
    typename Io<kX>::template Raw<kV> x[kScanTokens];
    const uint32_t cl = min(c, (uint32_t)(p.C - kV));  // lanes and tokens past the end load what is there and drop it
    if (p.N > 0)
#pragma unroll
        for (int i = 0; i < kScanTokens; ++i) {
            const int t = min(t0 + i, p.N - 1);
            z[i].load(row_at<kG>(p.gate, b, t, cl));
            x[i].load(row_at<kX>(p.x, b, t, cl));
        }
    const Places at = kPacked ? Places(p.offsets, p.sequences, t0, p.N, lane) : Places{};
    float entering[kV], a[kScanTokens][kV], h[kScanTokens][kV], A[kV], H[kV];
    if (!kPacked && k == 0 && wave == 0 && live) load_state<kV>(p.state_in, b, p.C, c, entering);
    else zero<kV>(entering);
#pragma unroll
    for (int v = 0; v < kV; ++v) { A[v] = 1.0f; H[v] = 0.0f; }
#pragma unroll
    for (int i = 0; i < kScanTokens; ++i) {
        if (i >= count) continue;
        const bool first = kPacked && (at.first >> i & 1);
        float enters[kV];
        if (first && live) load_state<kV>(p.state_in, at.of(i), p.C, c, enters);
        else zero<kV>(enters);
        z[i].get(a[i]);
        x[i].get(h[i]);
#pragma unroll
        for (int v = 0; v < kV; ++v) {
            float rest = 1.0f;
            decay<kMode>(a[i][v], a[i][v], rest);
            if (kMode == 2) h[i][v] *= rest;
            if (first) {
                // the only place where the state is read: as soon as this run is known state_out, which may be the
                // same memory, may be written
                h[i][v] = fmaf(a[i][v], enters[v], h[i][v]);
                H[v] = h[i][v];
            } else {
                H[v] = fmaf(a[i][v], H[v], h[i][v]);
                A[v] *= a[i][v];
            }
        }
    }
    float state[kV], after[kV];
    join_runs<kV, false, kPacked>(p, shared, block, k, wave, lane, live, A, H, kPacked && at.first != 0, entering, state, after);
#pragma unroll
    for (int i = 0; i < kScanTokens; ++i) {
        if (i >= count) continue;
        const bool first = kPacked && (at.first >> i & 1);
#pragma unroll
        for (int v = 0; v < kV; ++v) {
            state[v] = first ? h[i][v] : fmaf(a[i][v], state[v], h[i][v]);
            h[i][v] = state[v];
        }
        if (live && (!kPacked || (at.inside >> i & 1))) {
            store_channels<kX, kV>(p.out, b, t0 + i, c, h[i]);
            if (kPacked && (at.last >> i & 1)) store_state<kV>(p.state_out, at.of(i), p.C, c, h[i]);
        }
    }
    if (!live) return;
    if (kPacked) pass_on<kV>(p, p.state_in, p.state_out, k, wave, c);
    else if (k == p.tiles - 1 && wave == 0) store_state<kV>(p.state_out, b, p.C, c, after);
}

// The same from the last tile to the first.  The run of a wave maps the gradient that comes in from behind its last
// token to the one that goes out before its first.
template <int kX, int kG, int kMode, int kV, bool kPacked>
__global__ __launch_bounds__(64 * kScanWaves) void gated_scan_backward_kernel(GatedScanParams p) {
    __shared__ Shared<kV> shared;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int block, k;
    take_tile<kV>(p, shared, &block, &k);
    const int b = block / p.columns;
    const uint32_t c = (uint32_t)((block - b * p.columns) * 64 + lane) * kV;
    const bool live = c < (uint32_t)p.C;
    const int t0 = ((p.tiles - 1 - k) * p.waves + wave) * kScanTokens, count = min(max(p.N - t0, 0), kScanTokens);

    typename Io<kG>::template Raw<kV> z[kScanTokens];
    typename Io<kX>::template Raw<kV> dh[kScanTokens], h[kScanTokens], x[kScanTokens];  // h: of the token before
    const uint32_t cl = min(c, (uint32_t)(p.C - kV));  // lanes and tokens past the end load what is there and drop it
    if (p.N > 0)
#pragma unroll
        for (int i = 0; i < kScanTokens; ++i) {
            const int t = min(t0 + i, p.N - 1);
            z[i].load(row_at<kG>(p.gate, b, t, cl));
            dh[i].load(row_at<kX>(p.dh, b, t, cl));
            h[i].load(row_at<kX>(p.h, b, max(t - 1, 0), cl));
            if (kMode == 2) x[i].load(row_at<kX>(p.x, b, t, cl));
        }
    const Places at = kPacked ? Places(p.offsets, p.sequences, t0, p.N, lane) : Places{};
    float entering[kV], a[kScanTokens][kV], d[kScanTokens][kV], rest[kScanTokens][kV], A[kV], G[kV];
    if (!kPacked && k == 0 && wave == 0 && live) load_state<kV>(p.dstate_out, b, p.C, c, entering);
    else zero<kV>(entering);
#pragma unroll
    for (int v = 0; v < kV; ++v) { A[v] = 1.0f; G[v] = 0.0f; }
#pragma unroll
    for (int i = kScanTokens - 1; i >= 0; --i) {
        if (i >= count) continue;
        const bool last = kPacked && (at.last >> i & 1);
        float leaves[kV];
        if (last && live) load_state<kV>(p.dstate_out, at.of(i), p.C, c, leaves);
        else zero<kV>(leaves);
        z[i].get(a[i]);
        dh[i].get(d[i]);
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
    float g[kV], after[kV];  // g: the gradient that comes in from behind
    join_runs<kV, true, kPacked>(p, shared, block, k, wave, lane, live, A, G, kPacked && at.last != 0, entering, g, after);
#pragma unroll
    for (int i = kScanTokens - 1; i >= 0; --i) {
        if (i >= count || !live || (kPacked && !(at.inside >> i & 1))) continue;
        const bool last = kPacked && (at.last >> i & 1), first = kPacked ? (at.first >> i & 1) : t0 + i == 0;
        float before[kV], xi[kV], dx[kV], dgate[kV];
        if (first) load_state<kV>(p.state_in, kPacked ? at.of(i) : b, p.C, c, before);
        else h[i].get(before);
        if (kMode == 2) x[i].get(xi);
#pragma unroll
        for (int v = 0; v < kV; ++v) {
            const float D = last ? d[i][v] : d[i][v] + g[v];
            g[v] = a[i][v] * D;
            if (kMode == 0) { dgate[v] = D * before[v]; dx[v] = D; }
            else if (kMode == 1) { dgate[v] = g[v] * before[v]; dx[v] = D; }
            else { dgate[v] = g[v] * rest[i][v] * (before[v] - xi[v]); dx[v] = D * rest[i][v]; }
        }
        store_channels<kX, kV>(p.dx, b, t0 + i, c, dx);
        store_channels<kG, kV>(p.dgate, b, t0 + i, c, dgate);
        if (kPacked && first) store_state<kV>(p.dstate_in, at.of(i), p.C, c, g);
    }
    if (!live) return;
    if (kPacked) pass_on<kV>(p, p.dstate_out, p.dstate_in, k, wave, c);
    else if (k == p.tiles - 1 && wave == 0) store_state<kV>(p.dstate_in, b, p.C, c, after);
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
    const dim3 grid((unsigned)((long long)p.B * p.columns * p.tiles)), block(64 * (unsigned)p.waves);
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

// Column blocks, waves of a workgroup and tiles of N tokens; returns the bytes of workspace.
static size_t plan_scan(GatedScanParams* p) {
    const int v = p->vector >= 2 ? 2 : 1;
    p->columns = (p->C + 64 * v - 1) / (64 * v);
    const int need = (p->N + kScanTokens - 1) / kScanTokens;
    p->waves = need < 1 ? 1 : need < kScanWaves ? need : kScanWaves;  // no tokens: one that hands the states on
    const int tokens = p->waves * kScanTokens;
    p->tiles = p->N > 0 ? (p->N + tokens - 1) / tokens : 1;
    if (p->tiles == 1) return 0;
    const size_t lanes = (size_t)p->B * p->columns * 64 * p->tiles;
    return Board::kHeader + lanes * (8 * v + 8);
}

size_t gated_scan_workspace(int B, int N, int C, bool backward) {
    // the two channels a lane of aligned rows, or the one of others, whichever needs more
    size_t most = 0;
    for (int v = 1; v <= 2; ++v) {
        GatedScanParams p = {};
        p.B = B; p.N = N; p.C = C;
        p.vector = v;
        const size_t bytes = plan_scan(&p);
        if (bytes > most) most = bytes;
    }
    return most;
}

long long gated_scan_threads(int B, int N, int C, bool backward) {
    GatedScanParams p = {};
    p.B = B; p.N = N; p.C = C;
    p.vector = 1;
    plan_scan(&p);
    return (long long)p.B * p.columns * p.tiles * p.waves * 64;
}

static hipError_t launch_sequences(GatedScanParams& p, int elem, int gate_elem, int mode, int which, hipStream_t stream) {
    const size_t bytes = plan_scan(&p);
    if (bytes) {
        const size_t words = (bytes + 15) / 16;
        hipLaunchKernelGGL(gated_scan_clear_kernel, dim3((unsigned)((words + 255) / 256)), dim3(256), 0, stream,
                           static_cast<u32x4*>(p.workspace), words);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return launch_scan(p, elem, gate_elem, mode, which, stream);
}

hipError_t launch_gated_scan(GatedScanParams p, int elem, int gate_elem, int mode, hipStream_t stream) {
    return launch_sequences(p, elem, gate_elem, mode, 0, stream);
}

hipError_t launch_gated_scan_backward(GatedScanParams p, int elem, int gate_elem, int mode, hipStream_t stream) {
    return launch_sequences(p, elem, gate_elem, mode, 1, stream);
}

hipError_t launch_gated_step(GatedScanParams p, int elem, int gate_elem, int mode, hipStream_t stream) {
    return launch_scan(p, elem, gate_elem, mode, 2, stream);
}

}  // namespace leet
