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
// read once and outputs written once, which is what bounds it where there are many channels (a bf16 forward pass moves 6
// bytes a token and channel for some ten operations): N32768 C4096 with fp32 decays 205 us, 5.2 TB/s, where a copy of
// as many bytes runs at 5.1; B4 N4096 C2048 bf16 52 us, 3.9 TB/s.  Without the looks back that is 5 us less, without the
// tickets 1, without the kernel that clears the workspace 2 (parts left out; a trace, which keeps kernels apart, has 5.3 for
// that kernel and 48.8 for the scan).  Tried and slower: workgroups that stay and load the next tile during the look back
// (61 and 227 us: a tile's run is published only when the tile before it is done); a copy of both passes without branches
// for waves whose tokens are all there (51 us, but backward 105 instead of 92: registers).
//
// That holds while decays do not grow.  Ones above 1 in magnitude (none of a moving average's are) can take a product, and
// what it leaves of a zero state, out of fp32's range where the state itself is small: zeros with decays of 4 would be infinity
// times zero from token 64 on.  So where the decays above 1 that a wave holds multiply to more than kMostGrowth in any channel
// the tile is no run: its tokens are taken one after the other from the state before it, and the tiles behind it wait for that:
// some 8 us a tile of 112 tokens (every decay beyond that: B4 N4096 C2048 forward 305 us, N32768 C4096 2447; one token in a
// thousand of 20: 86 and 455).  Watching for them costs other calls 1 to 2 % (B4 N4096 C2048 52 -> 53 us, N32768 C4096 200 ->
// 205).
//
// Packed sequences: where a sequence begins, the run so far is cut off.  That is decided by the offsets alone, so it
// is the same for all channels and no arithmetic carries anything over (zero times an infinity would).
#include "leet_gated_scan.hpp"
#include "leet_io.hpp"

namespace leet {

// A tile: tokens of a wave, and waves of a workgroup that hold tokens (at most); one more wave links the tile to the others.
// Workgroups of 8, 12 or 16 waves spread evenly over the four SIMDs of a compute unit (B4 N4096 C2048 forward: 16 tokens x 7
// waves 57 us, 16 x 5 68, 12 x 9 71; backward 8 x 11 93, 8 x 9 102).  24 tokens x 7 waves, five waves a SIMD, are
// better where sequences are very long and worse elsewhere (16 | 24 tokens: N32768 C4096 178 157, B32 N512 C4096 82 97,
// N1000 C1024 12 14; of a moving average 186 187, 89 105, 16 20).
constexpr int kForwardTokens = 16, kBackwardTokens = 8, kMostWaves = 15;

// Of the tokens of a wave.  Fifteen waves' products then stay under 2^60, and rounding is multiplied by no more than the
// recurrence itself multiplies it by.
constexpr float kMostGrowth = 16.0f;

// A gate as it is kept between its two uses, in one register: the decay a itself, or for the moving average the smaller of
// a and 1 - a with the sign of the logit.  The larger one is what that leaves of 1, so both are as accurate as fp32 has
// them however near 0 or 1 they are.  The quotient e / (1 + e), e at most 1, is e times v_rcp_f32, which may be a step off,
// and what that leaves of e (exact in a fused multiply-add) times it once more: the nearest fp32 number for all 2^27.7 of e
// from 2^-26 on but five, whichever way the reciprocal is off, and for all below, where 1 + e is 1.  us uncorrected | with
// it | by a division: B4 N4096 C2048 bf16 forward 58 59 64, backward 89 89 113, packed N20011 C1001 fp16 59 59 64.
template <int kMode>
struct Gate {
    float g;

    __device__ __forceinline__ void set(float z) {
        if constexpr (kMode == 0) g = z;
        else if constexpr (kMode == 1) g = expf(z);
        else {
            const float e = expf(-fabsf(z));
            const float d = 1.0f + e, r = __builtin_amdgcn_rcpf(d), q = e * r;
            g = copysignf(fmaf(fmaf(-d, q, e), r, q), z);
        }
    }
    __device__ __forceinline__ bool below() const { return __builtin_bit_cast(int, g) < 0; }  // a logit below 0
    __device__ __forceinline__ float decay() const { return kMode != 2 ? g : below() ? -g : 1.0f - g; }
    __device__ __forceinline__ float rest() const { return kMode != 2 ? 1.0f : below() ? 1.0f + g : g; }
    // b of an input
    __device__ __forceinline__ float input(float x) const { return kMode != 2 ? x : rest() * x; }
};

// Where the tokens t0 .. t0 + kTokens - 1 lie among packed sequences.  Lane i < kTokens looks at token t0 + i.  A token's
// sequence is the last one that begins at or before it: of empty ones at one place the one behind them.
template <int kTokens>
struct Places {
    int sequence;          // this lane's token's
    uint32_t first, last;  // tokens that begin, end a sequence
    uint32_t inside;       // tokens that belong to one

    Places() = default;
    __device__ __forceinline__ Places(const int* offsets, int sequences, int t0, int N, int lane) {
        // the last s <= sequences with offsets[s] <= t0, 64 of the candidates at a time
        int s0 = 0, high = sequences;
        while (s0 < high) {
            const int step = (high - s0 + 63) / 64, s = s0 + (lane + 1) * step;
            s0 += step * __popcll(__ballot(s <= high && offsets[s <= high ? s : high] <= t0));
            high = min(high, s0 + step - 1);
        }
        const int end = min(t0 + kTokens, N);  // of the tokens that are there
        sequence = s0;
        first = last = inside = 0;
        if (s0 >= sequences || t0 >= N) return;  // behind the last sequence
        const uint32_t all = (uint32_t)((1u << (end - t0)) - 1u);
        const int begins = offsets[s0], ends = offsets[s0 + 1];
        if (ends >= end) {  // one sequence
            first = begins == t0 ? 1u : 0u;
            last = ends == end ? 1u << (end - t0 - 1) : 0u;
            inside = all;
            return;
        }
        // boundaries at or before the lane's token, 64 at a time
        for (int from = s0 + 1; from <= sequences; from += 64) {
            const int at = from + lane <= sequences ? offsets[from + lane] : 0x7fffffff;
#pragma unroll
            for (int i = 0; i < kTokens; ++i) {
                const int before = __popcll(__ballot(at <= t0 + i));
                sequence += lane == i ? before : 0;
            }
            if (__ballot(at < end) != ~0ull) break;
        }
        const int t = t0 + lane;
        const bool in = t < end && sequence < sequences;
        sequence = min(sequence, sequences - 1);
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
template <int kV>
__device__ __forceinline__ void zero(float* f) {
#pragma unroll
    for (int v = 0; v < kV; ++v) f[v] = 0.0f;
}
template <int kElem, int kV>
__device__ __forceinline__ void store_channels(const RowsOut& r, int b, long long t, uint32_t c, const float* f) {
    typename Io<kElem>::template Raw<kV> raw;
    raw.set(f);
    raw.store(r.data + (b * r.batch + t * r.token) * Io<kElem>::kBytes + c * Io<kElem>::kBytes);
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
constexpr uint32_t kUnset = 0xffffffffu;  // a NaN; a value with these bits is published as another one
constexpr uint32_t kCut = 0xfffffffeu;    // likewise: in the place of A, of a run that nothing before it reaches through

__device__ __forceinline__ uint32_t publishable(float f) {
    const uint32_t u = __builtin_bit_cast(uint32_t, f);
    return u >= kCut ? 0x7fc00000u : u;
}
__device__ __forceinline__ void publish(uint64_t* at, uint32_t lo, uint32_t hi) {
    __hip_atomic_store(at, (uint64_t)hi << 32 | lo, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint64_t look(const uint64_t* at) {
    return __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float low(uint64_t w) { return __builtin_bit_cast(float, (uint32_t)w); }
__device__ __forceinline__ float high(uint64_t w) { return __builtin_bit_cast(float, (uint32_t)(w >> 32)); }
__device__ __forceinline__ bool is_set(uint64_t w) { return (uint32_t)w != kUnset && (uint32_t)(w >> 32) != kUnset; }

// The state behind a run that was entered with s.
__device__ __forceinline__ float through(uint64_t run, float s) {
    return (uint32_t)run == kCut ? high(run) : fmaf(low(run), s, high(run));
}

// Workspace: kGroups lines, each with a ticket counter, then of every tile the runs of its channels (A, H: eight bytes a
// channel), then of every tile the inclusive states of its channels, four bytes a channel in pairs (a lone one: twice itself).
struct Board {
    uint64_t *runs, *states;
    long long tile;  // words of a tile's runs
    static constexpr int kGroups = 16, kLine = 32;  // most groups; 32-bit words of a line
    static constexpr size_t kHeader = kGroups * kLine * 4;

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
    __device__ __forceinline__ void publish_run(int k, bool cut, const float* A, const float* H) const {
#pragma unroll
        for (int v = 0; v < kV; ++v) publish(runs + k * tile + v, cut ? kCut : publishable(A[v]), publishable(H[v]));
    }
    template <int kV>
    __device__ __forceinline__ void publish_state(int k, const float* s) const {
        publish(states + k * (tile / kV), publishable(s[0]), publishable(s[kV - 1]));
    }

    // A window of what tiles k, k - 1, .. have published.  What is looked at in vain costs memory bandwidth: two, four and
    // eight tiles at a time, B4 N4096 C2048 (64 chains) 52, 54 and 55 us.  That is decided by where many chains look: one
    // sequence of 20000 tokens, moving average, C128 (one chain) 40 37 57, C512 (4) 44 40 69, C1024 (8) 48 49 82, C2048 70 83 100.
    template <int kV>
    struct Window {
        static constexpr int kTiles = 2;
        uint64_t run[kTiles][kV], whole[kTiles];
        int runs;    // so many, from tile k on, have published their runs ..
        bool ended;  // .. and the next one its state

        __device__ __forceinline__ void load(const Board& board, int k, bool live) {
#pragma unroll
            for (int u = 0; u < kTiles; ++u) {
                const int j = max(k - u, 0);
                whole[u] = live ? look(board.states + j * (board.tile / kV)) : 0;
#pragma unroll
                for (int v = 0; v < kV; ++v) run[u][v] = live ? look(board.runs + j * board.tile + v) : 0;
            }
            runs = 0;
            ended = false;
#pragma unroll
            for (int u = 0; u < kTiles; ++u) {
                bool set = true;
#pragma unroll
                for (int v = 0; v < kV; ++v) set = set && is_set(run[u][v]);
                if (runs == u && !ended) {
                    if (__all(is_set(whole[u]))) ended = true;
                    else if (__all(set)) ++runs;  // never the first tile, which publishes its state alone
                }
            }
        }
        // from the state behind the tile after the window's runs (or the one that ended it) to the state behind tile k
        __device__ __forceinline__ void fold(float* state) const {
#pragma unroll
            for (int u = kTiles - 1; u >= 0; --u)
#pragma unroll
                for (int v = 0; v < kV; ++v) {
                    if (ended && u == runs) state[v] = v ? high(whole[u]) : low(whole[u]);
                    if (u < runs) state[v] = through(run[u][v], state[v]);
                }
        }
    };

    // The state behind tile k of the chain: looks back until it meets a tile whose state is known, waiting for those that
    // have published nothing, and goes forward from there over the runs.  So it is the same chain of fused multiply-adds
    // whatever was known when: results do not depend on timing.  Every wait ends: a tile publishes its run (the first tile
    // its state) without waiting for anything, or, where its tokens are taken one after the other, its state after waiting
    // for tiles before it alone; and tiles are taken in the order of the chain, so all that are waited for belong to
    // workgroups that are running already.  That holds while the workspace is this launch's alone; kPatience
    // ends the wait, with NaN for the state, where it is not: some seconds of looks, a million times what a wait takes.
    static constexpr int kPatience = 1 << 22;
    template <int kV>
    __device__ __forceinline__ void state_behind(int k, bool live, float* state) const {
        constexpr int kTiles = Window<kV>::kTiles;
        Window<kV> near, far;
        int looks = 0;
        do near.load(*this, k, live);
        while (!near.ended && near.runs < kTiles && ++looks < kPatience);
        zero<kV>(state);
        if (!near.ended) {
            int j = k - kTiles;
            while (looks < kPatience) {
                far.load(*this, j, live);
                if (far.ended) break;
                j -= far.runs;
                ++looks;
            }
            if (looks >= kPatience) {
#pragma unroll
                for (int v = 0; v < kV; ++v) state[v] = __builtin_bit_cast(float, 0x7fc00000u);
                return;
            }
            far.fold(state);
            // tiles j + 1 .. k - kTiles, whose runs have all been seen; the last window of them may be a short one
            for (j += kTiles; j < k; j += kTiles) {
                const int top = min(j, k - kTiles), skip = j - top;
                far.load(*this, top, live);
                far.ended = false;
                far.runs = kTiles - skip;
                far.fold(state);
            }
        }
        near.fold(state);
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
    float A[kMostWaves][64 * kV], H[kMostWaves][64 * kV];  // the waves' runs
    int cut[kMostWaves];    // a sequence begins (backward: ends) in the run: what came before does not reach behind it
    int grows[kMostWaves];  // by more than kMostGrowth
    float carry[64 * kV];
    int serial;  // one of the runs does: the waves go on one after the other
    unsigned ticket;
};

// The tile of a workgroup: tile k of the chain of column block `block` (of all batch entries).  Tiles are taken in the order
// in which workgroups start, whatever that is: workgroup l to start of group g takes tile l groups + g of all, counted
// chain by chain first and along the chains last.  groups divides the number of chains, so all tiles of a chain belong to
// one group, and every tile before this one on its chain has been taken.  Eight workgroups in a row, which go to the eight
// XCDs, belong to one group: chains then advance together and rows are read whole.  us with one counter | sixteen groups |
// one counter for every chain | sixteen groups of workgroups equal modulo 16, two for each XCD: B4 N4096 C2048 bf16
// 53 51 52 52, N32768 C4096 197 196 221 221, packed N20011 C1001 fp16 57 54 53 54.  False: a workgroup beyond the last tile.
template <class S>
__device__ __forceinline__ bool take_tile(const GatedScanParams& p, S& shared, int* block, int* k) {
    const unsigned blocks = (unsigned)p.B * (unsigned)p.columns;
    unsigned tile = blockIdx.x;
    if (p.tiles > 1) {
        const unsigned group = (blockIdx.x >> 3) % (unsigned)p.groups;
        if (threadIdx.x == 0) shared.ticket = atomicAdd(static_cast<unsigned*>(p.workspace) + group * Board::kLine, 1u);
        __syncthreads();
        tile = (unsigned)__builtin_amdgcn_readfirstlane((int)shared.ticket) * p.groups + group;
    }
    *k = (int)(tile / blocks);
    *block = (int)(tile - (unsigned)*k * blocks);
    return *k < p.tiles;
}

// The wave behind the data waves links the tile to the others: it joins the waves' runs, publishes, looks back, and leaves
// the state before the tile in shared.carry.  The registers that looking back takes are then not beside a tile's data.
// Of a tile whose tokens are taken one after the other it publishes the state alone, when the last data wave has left it in
// shared.carry.
// kBackward: the chain goes from the last wave to the first.
template <int kMode, int kV, bool kBackward, bool kPacked, class S>
__device__ __forceinline__ void link_tile(const GatedScanParams& p, S& shared, int block, int k, int lane, bool live,
                                          const float* state_in, float* state_out, int b, uint32_t c) {
    float carry[kV], A[kV], H[kV];
    if (!kPacked && k == 0 && live) load_state<kV>(state_in, b, p.C, c, carry);
    else zero<kV>(carry);
    __syncthreads();  // the waves' runs are there
    bool cut = false;
    int grows = 0;
#pragma unroll
    for (int v = 0; v < kV; ++v) { A[v] = 1.0f; H[v] = 0.0f; }
    for (int i = 0; i < p.waves; ++i) {
        const int w = kBackward ? p.waves - 1 - i : i;
        const bool here = kPacked && shared.cut[w];
        cut = cut || here;
        if (kMode != 2) grows |= shared.grows[w];
#pragma unroll
        for (int v = 0; v < kV; ++v) {
            const float Hw = shared.H[w][lane * kV + v], Aw = shared.A[w][lane * kV + v];
            H[v] = here ? Hw : fmaf(Aw, H[v], Hw);
            A[v] *= Aw;
        }
    }
    const bool serial = kMode != 2 && __builtin_expect(__builtin_amdgcn_readfirstlane(grows), 0);
    const Board board = Board::of<kV>(p, block, lane);
    if (k > 0) {
        if (live && !serial) board.publish_run<kV>(k, cut, A, H);
        if (live && !serial && cut) board.publish_state<kV>(k, H);
        board.state_behind<kV>(k - 1, live, carry);
    }
#pragma unroll
    for (int v = 0; v < kV; ++v) shared.carry[lane * kV + v] = carry[v];
    if (kMode != 2 && lane == 0) shared.serial = serial;
    __syncthreads();  // the state before the tile is there
#pragma unroll
    for (int v = 0; v < kV; ++v) H[v] = cut ? H[v] : fmaf(A[v], carry[v], H[v]);
    if (__builtin_expect(serial, 0)) {
        for (int i = 0; i < p.waves; ++i) __syncthreads();  // the data waves, one after the other
#pragma unroll
        for (int v = 0; v < kV; ++v) H[v] = shared.carry[lane * kV + v];
    }
    if (live && k + 1 < p.tiles && (k == 0 || !cut || serial)) board.publish_state<kV>(k, H);
    if (!kPacked && live && k == p.tiles - 1) store_state<kV>(state_out, b, p.C, c, H);
}

// A data wave's part: its run goes to the others; before[] receives the state before it.  True: the waves go on one after
// the other, and this one has to hand its state on.
template <int kMode, int kV, bool kBackward, bool kPacked, class S>
__device__ __forceinline__ bool join_runs(const GatedScanParams& p, S& shared, int wave, int lane, const float* A,
                                          const float* H, bool cut, bool grows, float* before) {
#pragma unroll
    for (int v = 0; v < kV; ++v) {
        shared.A[wave][lane * kV + v] = A[v];
        shared.H[wave][lane * kV + v] = H[v];
    }
    if (kPacked && lane == 0) shared.cut[wave] = cut;
    if (kMode != 2 && lane == 0) shared.grows[wave] = grows;
    __syncthreads();
    float beforeA[kV];
#pragma unroll
    for (int v = 0; v < kV; ++v) { beforeA[v] = 1.0f; before[v] = 0.0f; }
    bool cut_before = false;
    const int ahead = kBackward ? p.waves - 1 - wave : wave;  // runs that come before this wave's
    for (int i = 0; i < ahead; ++i) {
        const int w = kBackward ? p.waves - 1 - i : i;
        const bool here = kPacked && shared.cut[w];
        cut_before = cut_before || here;
#pragma unroll
        for (int v = 0; v < kV; ++v) {
            const float Hw = shared.H[w][lane * kV + v], Aw = shared.A[w][lane * kV + v];
            before[v] = here ? Hw : fmaf(Aw, before[v], Hw);
            beforeA[v] *= Aw;
        }
    }
    __syncthreads();
    if (kMode != 2 && __builtin_expect(__builtin_amdgcn_readfirstlane(shared.serial), 0)) {
        for (int i = 0; i < ahead; ++i) __syncthreads();
#pragma unroll
        for (int v = 0; v < kV; ++v) before[v] = shared.carry[lane * kV + v];
        return true;
    }
#pragma unroll
    for (int v = 0; v < kV; ++v)
        before[v] = cut_before ? before[v] : fmaf(beforeA[v], shared.carry[lane * kV + v], before[v]);
    return false;
}

// The end of a data wave's turn in a tile whose waves go on one after the other: its state is the next one's.
template <int kV, bool kBackward, class S>
__device__ __forceinline__ void hand_on(const GatedScanParams& p, S& shared, int wave, int lane, const float* state) {
#pragma unroll
    for (int v = 0; v < kV; ++v) shared.carry[lane * kV + v] = state[v];
    for (int i = kBackward ? p.waves - 1 - wave : wave; i < p.waves; ++i) __syncthreads();
}

// The first channel of a lane.  The last pair of an odd number of channels begins one channel early: that channel is then
// computed and stored twice, the same both times.  The lane before does so too, and has to be in the same wave: where states
// are updated in place, another workgroup could have written that channel's before this one reads it.  So where the last
// column has one channel, it takes the last pair of the column before it over.  Lanes past the end (false) load what the last
// pair loads.
template <int kV>
__device__ __forceinline__ bool channel_of(const GatedScanParams& p, int column, int lane, uint32_t* c) {
    int at = (column * 64 + lane) * kV;
    bool live = true;
    if (kV == 2 && p.C % (64 * kV) == 1) {
        if (column == p.columns - 1) at -= kV;
        else live = column < p.columns - 2 || lane < 63;
    }
    *c = min((uint32_t)at, (uint32_t)(p.C - kV));
    return live && at < p.C;
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

// Workgroup = one tile of waves * kTokens tokens x 64 kV channels of one batch entry.  Six waves a SIMD, three workgroups of
// eight waves a unit, where the inputs' registers allow it; the compiler stays under 65 registers there, so it is four
// workgroups (us with bounds of six and four: B4 N4096 C2048 50 51, its sigmoid 55 59, N32768 C4096 sigmoid 185 207; with
// fp32 gates 206 200).
template <int kX, int kG, int kMode, int kV, bool kPacked>
__global__ __launch_bounds__(64 * (kMostWaves + 1), kX != 0 && kG != 0 && !kPacked ? 6 : 4) void gated_scan_kernel(GatedScanParams p) {
    constexpr int kTokens = kForwardTokens;
    __shared__ Shared<kV> shared;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int block, k;
    if (!take_tile(p, shared, &block, &k)) return;
    const int b = block / p.columns;
    uint32_t c;
    const bool live = channel_of<kV>(p, block - b * p.columns, lane, &c);
    if (wave == p.waves) {
        link_tile<kMode, kV, false, kPacked>(p, shared, block, k, lane, live, p.state_in, p.state_out, b, c);
        return;
    }
    const int t0 = (k * p.waves + wave) * kTokens, count = min(max(p.N - t0, 0), kTokens);

    typename Io<kG>::template Raw<kV> z[kTokens];
    typename Io<kX>::template Raw<kV> x[kTokens];
    if (p.N > 0)  // tokens past the end load what is there and drop it
#pragma unroll
        for (int i = 0; i < kTokens; ++i) {
            const int t = min(t0 + i, p.N - 1);
            z[i].load(row_at<kG>(p.gate, b, t, c));
            x[i].load(row_at<kX>(p.x, b, t, c));
        }
    const Places<kTokens> at = kPacked ? Places<kTokens>(p.offsets, p.sequences, t0, p.N, lane) : Places<kTokens>{};
    Gate<kMode> g[kTokens][kV];
    // b with what enters a sequence; without packed sequences it is the input, kept as it was loaded (half the registers:
    // three workgroups a compute unit instead of two)
    float h[kPacked ? kTokens : 1][kV];
    float A[kV], H[kV];
    float growth = 1.0f;  // product of the decays above 1, the larger of the channels'
#pragma unroll
    for (int v = 0; v < kV; ++v) { A[v] = 1.0f; H[v] = 0.0f; }
#pragma unroll
    for (int i = 0; i < kTokens; ++i) {
        if (i >= count) continue;
        const bool first = kPacked && (at.first >> i & 1);
        float enters[kV];
        if (first && live) load_state<kV>(p.state_in, at.of(i), p.C, c, enters);
        else zero<kV>(enters);
        float zi[kV], xi[kV];
        z[i].get(zi);
        x[i].get(xi);
        float largest = 1.0f;
#pragma unroll
        for (int v = 0; v < kV; ++v) {
            g[i][v].set(zi[v]);
            // one channel's exponential and quotient after the other's: interleaved they take 65 to 67 registers instead of
            // 63, three workgroups a unit instead of four (B4 N4096 C2048 bf16 sigmoid 61 us instead of 59)
            if (kMode != 0 && v + 1 < kV) asm volatile("" : "+v"(g[i][v].g), "+v"(zi[v + 1]));
            const float a = g[i][v].decay();
            float b = g[i][v].input(xi[v]);
            largest = fmaxf(largest, fabsf(a));
            if (first) {
                // the only place where the state is read: as soon as this run is known state_out, which may be the
                // same memory, may be written
                b = fmaf(a, enters[v], b);
                H[v] = b;
            } else {
                H[v] = fmaf(a, H[v], b);
                A[v] *= a;
            }
            if (kPacked) h[i][v] = b;
        }
        growth *= largest;
    }
    float state[kV];
    const bool serial = join_runs<kMode, kV, false, kPacked>(p, shared, wave, lane, A, H, kPacked && at.first != 0,
                                                             kMode != 2 && __any(growth > kMostGrowth) && (!kPacked || at.inside), state);
#pragma unroll
    for (int i = 0; i < kTokens; ++i) {
        if (i >= count) continue;
        const bool first = kPacked && (at.first >> i & 1);
        float xi[kV];
        if (!kPacked) x[i].get(xi);
#pragma unroll
        for (int v = 0; v < kV; ++v) {
            const float b = kPacked ? h[i][v] : g[i][v].input(xi[v]);
            state[v] = first ? b : fmaf(g[i][v].decay(), state[v], b);
        }
        if (live && (!kPacked || (at.inside >> i & 1))) {
            store_channels<kX, kV>(p.out, b, t0 + i, c, state);
            if (kPacked && (at.last >> i & 1)) store_state<kV>(p.state_out, at.of(i), p.C, c, state);
        }
    }
    if (__builtin_expect(serial, 0)) hand_on<kV, false>(p, shared, wave, lane, state);
    if (kPacked && live) pass_on<kV>(p, p.state_in, p.state_out, k, wave, c);
}

// The same from the last tile to the first.  The run of a wave maps the gradient that comes in from behind its last
// token to the one that goes out before its first.
template <int kX, int kG, int kMode, int kV, bool kPacked>
__global__ __launch_bounds__(64 * (kMostWaves + 1)) void gated_scan_backward_kernel(GatedScanParams p) {
    constexpr int kTokens = kBackwardTokens;
    __shared__ Shared<kV> shared;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int block, k;
    if (!take_tile(p, shared, &block, &k)) return;
    const int b = block / p.columns;
    uint32_t c;
    const bool live = channel_of<kV>(p, block - b * p.columns, lane, &c);
    if (wave == p.waves) {
        link_tile<kMode, kV, true, kPacked>(p, shared, block, k, lane, live, p.dstate_out, p.dstate_in, b, c);
        return;
    }
    const int t0 = ((p.tiles - 1 - k) * p.waves + wave) * kTokens, count = min(max(p.N - t0, 0), kTokens);

    typename Io<kG>::template Raw<kV> z[kTokens];
    typename Io<kX>::template Raw<kV> dh[kTokens], h[kTokens], x[kTokens];  // h: of the token before
    if (p.N > 0)  // tokens past the end load what is there and drop it
#pragma unroll
        for (int i = 0; i < kTokens; ++i) {
            const int t = min(t0 + i, p.N - 1);
            z[i].load(row_at<kG>(p.gate, b, t, c));
            dh[i].load(row_at<kX>(p.dh, b, t, c));
            h[i].load(row_at<kX>(p.h, b, max(t - 1, 0), c));
            if (kMode == 2) x[i].load(row_at<kX>(p.x, b, t, c));
        }
    const Places<kTokens> at = kPacked ? Places<kTokens>(p.offsets, p.sequences, t0, p.N, lane) : Places<kTokens>{};
    Gate<kMode> gate[kTokens][kV];
    float d[kTokens][kV], A[kV], G[kV];
    float growth = 1.0f;  // product of the decays above 1, the larger of the channels'
#pragma unroll
    for (int v = 0; v < kV; ++v) { A[v] = 1.0f; G[v] = 0.0f; }
#pragma unroll
    for (int i = kTokens - 1; i >= 0; --i) {
        if (i >= count) continue;
        const bool last = kPacked && (at.last >> i & 1);
        float leaves[kV];
        if (last && live) load_state<kV>(p.dstate_out, at.of(i), p.C, c, leaves);
        else zero<kV>(leaves);
        float zi[kV];
        z[i].get(zi);
        dh[i].get(d[i]);
        float largest = 1.0f;
#pragma unroll
        for (int v = 0; v < kV; ++v) {
            gate[i][v].set(zi[v]);
            const float a = gate[i][v].decay();
            largest = fmaxf(largest, fabsf(a));
            if (last) {
                d[i][v] += leaves[v];
                G[v] = a * d[i][v];
            } else {
                G[v] = a * (d[i][v] + G[v]);
                A[v] *= a;
            }
        }
        growth *= largest;
    }
    float g[kV];  // the gradient that comes in from behind
    const bool serial = join_runs<kMode, kV, true, kPacked>(p, shared, wave, lane, A, G, kPacked && at.last != 0,
                                                            kMode != 2 && __any(growth > kMostGrowth) && (!kPacked || at.inside), g);
#pragma unroll
    for (int i = kTokens - 1; i >= 0; --i) {
        if (i >= count || !live || (kPacked && !(at.inside >> i & 1))) continue;
        const bool last = kPacked && (at.last >> i & 1), first = kPacked ? (at.first >> i & 1) : t0 + i == 0;
        float before[kV], xi[kV], dx[kV], dgate[kV];
        if (first) load_state<kV>(p.state_in, kPacked ? at.of(i) : b, p.C, c, before);
        else h[i].get(before);
        if (kMode == 2) x[i].get(xi);
#pragma unroll
        for (int v = 0; v < kV; ++v) {
            const float D = last ? d[i][v] : d[i][v] + g[v];
            const float rest = gate[i][v].rest();
            g[v] = gate[i][v].decay() * D;
            if (kMode == 0) { dgate[v] = D * before[v]; dx[v] = D; }
            else if (kMode == 1) { dgate[v] = g[v] * before[v]; dx[v] = D; }
            else { dgate[v] = g[v] * rest * (before[v] - xi[v]); dx[v] = D * rest; }
        }
        store_channels<kX, kV>(p.dx, b, t0 + i, c, dx);
        store_channels<kG, kV>(p.dgate, b, t0 + i, c, dgate);
        if (kPacked && first) store_state<kV>(p.dstate_in, at.of(i), p.C, c, g);
    }
    if (__builtin_expect(serial, 0)) hand_on<kV, true>(p, shared, wave, lane, g);
    if (kPacked && live) pass_on<kV>(p, p.dstate_out, p.dstate_in, k, wave, c);
}

// One token of every sequence: state <- a state + b, out = state.  One thread per kV channels.  Sequences are counted
// without a sign: a stride of the grid behind the last of 2^31 - 1 is still a number.
template <int kX, int kG, int kMode, int kV>
__global__ __launch_bounds__(256) void gated_step_kernel(GatedScanParams p) {
    const uint32_t c = (blockIdx.x * 256 + threadIdx.x) * kV;
    if (c >= (uint32_t)p.C) return;
    for (unsigned b = blockIdx.y; b < (unsigned)p.B; b += gridDim.y) {
        float z[kV], x[kV], s[kV];
        Io<kG>::template load<kV>(row_at<kG>(p.gate, (int)b, 0, c), z);
        Io<kX>::template load<kV>(row_at<kX>(p.x, (int)b, 0, c), x);
        char* state = reinterpret_cast<char*>(p.state_out + (size_t)b * p.C + c);
        Io<0>::load<kV>(state, s);
#pragma unroll
        for (int v = 0; v < kV; ++v) {
            Gate<kMode> g;
            g.set(z[v]);
            s[v] = fmaf(g.decay(), s[v], g.input(x[v]));
        }
        Io<0>::store<kV>(state, s);
        Io<kX>::template store<kV>(p.out.data + (b * p.out.batch + c) * Io<kX>::kBytes, s);
    }
}

// which: 0 forward, 1 backward
template <int kX, int kG, int kMode, int kV>
static void launch_scan_v(const GatedScanParams& p, int which, hipStream_t stream) {
    // whole rounds of the groups: each is as many workgroups as the others
    const long long all = (long long)p.B * p.columns * p.tiles, round = p.tiles > 1 ? 8LL * p.groups : 1;
    const dim3 grid((unsigned)((all + round - 1) / round * round)), block(64 * (unsigned)(p.waves + 1));
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
    } else if (p.C > 1) launch_scan_v<kX, kG, kMode, 2>(p, which, stream);
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

// Waves of a workgroup that hold tokens.  A chain advances a tile every 0.3 us, so where there are few chains long tiles
// count; else that several workgroups fit a compute unit.  us with 7 | 11 | 15 waves, bf16: forward N20000 C1024 (8 chains)
// 65 47 43, C2048 (16) 80 71 69, B2 N4096 C2048 (32) 31 32 33, B4 (64) 50 58 61, N32768 C4096 (32) 176 200 194; backward
// C1024 125 86 72, B4 N4096 C2048 79 76 74, N32768 C4096 313 267 253.
// Packed sequences count as chains of their own, however long they are: their offsets lie on the device.  bf16 moving average,
// 20011 tokens, 7 | 15 waves: 37 equal sequences forward C128 18 21, C1001 56 61, C2048 92 115, backward C128 21 19, C1001 79
// 96, C2048 126 165; one long sequence and 36 of ten tokens forward C128 64 43, C1001 75 65, C2048 97 114, backward C128 111 62,
// C1001 137 97, C2048 162 156.  So it costs a third where nearly all tokens are one sequence's and channels are few (forward),
// and up to a quarter where sequences are equal and channels many (backward).
constexpr int kForwardWaves = 7;
static int waves_of(const GatedScanParams& p, bool backward) {
    const long long chains = (long long)p.B * p.columns * (p.offsets ? p.sequences : 1);
    return !backward && chains > 16 ? kForwardWaves : kMostWaves;
}

// Column blocks, waves of a workgroup and tiles of N tokens; returns the bytes of workspace.
// most: the waves, or 0 for what the sizes ask for; the fewest give the most bytes, room for any sequences.
static size_t plan_scan(GatedScanParams* p, bool backward, int most) {
    const int v = p->C > 1 ? 2 : 1;
    const int tokens = backward ? kBackwardTokens : kForwardTokens;
    p->columns = (p->C + 64 * v - 1) / (64 * v);
    const long long chains = (long long)p->B * p->columns;
    const int need = (p->N + tokens - 1) / tokens;
    if (most == 0) most = waves_of(*p, backward);
    p->waves = need < 1 ? 1 : need < most ? need : most;  // no tokens: one that hands the states on
    p->tiles = need < 1 ? 1 : (need + p->waves - 1) / p->waves;
    for (p->groups = Board::kGroups; chains % p->groups != 0;) p->groups /= 2;
    return p->tiles == 1 ? 0 : Board::kHeader + (size_t)chains * 64 * p->tiles * (8 * v + 8);
}

size_t gated_scan_workspace(int B, int N, int C, bool backward) {
    GatedScanParams p = {};
    p.B = B; p.N = N; p.C = C;
    return plan_scan(&p, backward, backward ? kMostWaves : kForwardWaves);
}

long long gated_scan_threads(int B, int N, int C, bool backward) {
    GatedScanParams p = {};
    p.B = B; p.N = N; p.C = C;
    plan_scan(&p, backward, backward ? kMostWaves : kForwardWaves);
    const long long chains = (long long)p.B * p.columns, wide = (kMostWaves + 1) * 64;
    if (chains >= 1LL << 22) return chains * wide;  // too many by themselves; times the tiles might not fit
    return (chains * p.tiles + Board::kGroups * 8) * wide;
}

static hipError_t launch_sequences(GatedScanParams& p, int elem, int gate_elem, int mode, int which, hipStream_t stream) {
    const size_t bytes = plan_scan(&p, which != 0, 0);
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
