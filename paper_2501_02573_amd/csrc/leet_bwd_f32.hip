// Backward pass of the decayed causal linear attention for fp32 inputs (gfx950, v_mfma_f32_16x16x4_f32: true fp32 products).
//
// The walks of leet_bwd_16bit.hip: out = ((X Y^T) .* M) Z in the order of the tokens (dQ) or the reversed one (dK, dV),
//
//     O_t     = ((X_t Y_t^T) .* D) Z_t + Lam (X_t S_t)       D[i][j] = gamma^(i-j), i >= j
//     S_{t+1} = gamma^L S_t + (Gam Y_t)^T Z_t
//
// Bound by the matrix instructions: at width 128 a chunk of a role is 5.5 MFLOP, 9 us of one compute unit's rate, and takes 11.8
// (76 %): the barriers and the first operands of each product.  B2 H8 N2047 d128 with states: pre-pass, scan and walk 31, 12 and
// 116 us.  Wave w owns 16 columns of O and S; the ten
// 16 x 16 score tiles on and below the diagonal are each formed once a workgroup and handed on through LDS.
//
// MFMA conventions (16x16x4 fp32): an A (B) operand is one float per lane: lane l holds row (column) l%16 and contraction
// slot q = l/16; an accumulator holds, in lane l, column l%16 and, in register r, row 4q + r.  Everything is computed
// transposed (lane = token), so that an accumulator register of one product is directly an operand of the next.
#include "leet_backward.hpp"
#include "leet_common.hpp"

namespace leet {
namespace bwd {

template <int D, bool kOut>
struct Smem32 {
    static constexpr int RS = D + 4;  // padded row stride (floats)
    float x[kOut ? kChunk * RS : 4];
    float y[kChunk * RS];
    float z[kChunk * RS];
    f32x4 pfrag[kOut ? 10 : 1][64];   // masked score tiles: [tile][lane], registers 0..3
    float pw[kChunk + 4];             // gamma^n, n = 0..64
};

// The ten score tiles (it >= jt) in production order.
__device__ __forceinline__ constexpr int tile32_it(int n) { return n < 1 ? 0 : n < 3 ? 1 : n < 6 ? 2 : 3; }
__device__ __forceinline__ constexpr int tile32_jt(int n) { return n - (tile32_it(n) * (tile32_it(n) + 1)) / 2; }

// kOut = true: outputs and state.  kOut = false: state only, of every segment but the last, started from zero.
template <int D, bool kOut>
__global__ __launch_bounds__(D * 4, D > 64 ? 1 : 2) void walk32_kernel(BwdParams p) {
    constexpr int NT = D * 4;                  // threads: one wave per 16 columns
    constexpr int NW = D / 16;                 // waves
    constexpr int DT = D / 16;                 // 16-row tiles of the state
    constexpr int RS = Smem32<D, kOut>::RS;
    constexpr int PR = D / 4;                  // 16-byte pieces per row
    constexpr int NLOAD = kChunk * PR / NT;    // pieces per thread per tensor
    constexpr int ROWS_PER_PASS = NT / PR;
    constexpr int NSLOT = (10 + NW - 1) / NW;  // score tiles per wave, at most
    __shared__ __attribute__((aligned(16))) Smem32<D, kOut> sm;

    const int tid = threadIdx.x;
    const int w = tid >> 6, l = tid & 63, ln = l & 15, qd = l >> 4;
    const int nseg = kOut ? p.nseg : p.nseg - 1;
    const int slot = blockIdx.x >> 3, which = slot % p.roles, unit = (slot / p.roles) * 8 + (blockIdx.x & 7);
    if (unit >= p.BH * nseg) return;
    const BwdRole& role = p.role[which];
    const bool rev = role.reversed != 0;
    const int bh = unit / nseg;
    const int seg = rev ? nseg - 1 - unit % nseg : unit % nseg;
    const int h = bh % p.H;
    const int later = rev ? 0 : 1;

    const int tok_begin = seg * p.seg_chunks * kChunk;
    const int tok_end = (seg == p.nseg - 1) ? p.N : tok_begin + p.seg_chunks * kChunk;
    const int nchunks = (tok_end - tok_begin + kChunk - 1) / kChunk;

    // token t of the walk is row t, or N - 1 - t, of the tensors
    const size_t first = ((size_t)bh * p.N + (rev ? p.N - 1 : 0)) * D;
    const ptrdiff_t row = rev ? -D : D;
    const float* xb = static_cast<const float*>(role.x) + first;
    const float* yb = static_cast<const float*>(role.y) + first;
    const float* zb = static_cast<const float*>(role.z) + first;
    float* ob = static_cast<float*>(role.out) + first;

    const double gd = p.gamma ? (double)p.gamma[h] : 1.0;
    for (int n = tid; n <= kChunk; n += NT) sm.pw[n] = (float)pow_int(gd, n);

    // state slice: S[t][r] = S[dk = 16t + 4q + r][c = 16w + ln]
    f32x4 S[DT];
    const int c_own = 16 * w + ln;
#pragma unroll
    for (int t = 0; t < DT; ++t) S[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (kOut && seg > 0) {
        const float* src = role.slots + ((size_t)bh * (p.nseg - 1) + seg - 1) * D * D + (size_t)c_own * role.slot_col;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) S[t][r] = src[(16 * t + 4 * qd + r) * role.slot_row];
    }
    if (kOut && role.enter) {
        const float* src = role.enter + (size_t)bh * D * D + (size_t)c_own * role.enter_col;
        const float left = (float)pow_int(gd, tok_begin);
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) S[t][r] += left * src[(16 * t + 4 * qd + r) * role.enter_row];
    }
    __syncthreads();  // table visible

    // per-lane constants of the walk
    f32x4 wgt[NSLOT];   // decay weights of the score tiles this wave produces
    float gam[16];      // Gam of the tokens j = 16jt + 4q + r that this lane feeds to the state
#pragma unroll
    for (int n = 0; n < 10; ++n) {
        if (n % NW != w) continue;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int d = 16 * (tile32_it(n) - tile32_jt(n)) + ln - (4 * qd + r);  // i - j
            wgt[n / NW][r] = (d >= 0) ? sm.pw[max(d, 0)] : 0.0f;
        }
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) gam[e] = sm.pw[kChunk - later - (16 * (e >> 2) + 4 * qd + (e & 3))];

    // staging: piece r of this thread is row ROWS_PER_PASS*r + tid/PR, floats 4(tid%PR)..+3
    const int j0 = tid / PR, cc = tid % PR;
    f32x4 rx[NLOAD], ry[NLOAD], rz[NLOAD];
    auto prefetch = [&](int tok0) {
        const int shift = max(0, tok0 + kChunk - tok_end);  // rows [0, shift) of the tile stay zero
#pragma unroll
        for (int r = 0; r < NLOAD; ++r) {
            const int j = ROWS_PER_PASS * r + j0;
            const bool ok = j >= shift;
            const ptrdiff_t off = (tok0 - shift + j) * row + cc * 4;
            const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
            if (kOut) rx[r] = ok ? *reinterpret_cast<const f32x4*>(xb + off) : zero;
            ry[r] = ok ? *reinterpret_cast<const f32x4*>(yb + off) : zero;
            rz[r] = ok ? *reinterpret_cast<const f32x4*>(zb + off) : zero;
        }
    };

    prefetch(tok_begin);

    for (int t = 0; t < nchunks; ++t) {
        const int tok0 = tok_begin + t * kChunk;
        const int Lc = min(kChunk, tok_end - tok0);
        const int shift = kChunk - Lc;  // a ragged last chunk is right-aligned in the tile, rows above are zero

        if (t > 0) __syncthreads();  // everyone is done reading the previous chunk's tiles and score fragments
#pragma unroll
        for (int r = 0; r < NLOAD; ++r) {
            const int j = ROWS_PER_PASS * r + j0;
            if (kOut) *reinterpret_cast<f32x4*>(&sm.x[j * RS + cc * 4]) = rx[r];
            *reinterpret_cast<f32x4*>(&sm.y[j * RS + cc * 4]) = ry[r];
            *reinterpret_cast<f32x4*>(&sm.z[j * RS + cc * 4]) = rz[r];
        }
        __syncthreads();
        if (t + 1 < nchunks) prefetch(tok0 + kChunk);  // in flight during the MFMA work below

        f32x4 o[4];
        if (kOut) {
            // P^T = Y X^T, masked, for the score tiles this wave produces
#pragma unroll
            for (int n = 0; n < 10; ++n) {
                if (n % NW != w) continue;
                f32x4 acc = {0.f, 0.f, 0.f, 0.f};
                const float* yrow = &sm.y[(16 * tile32_jt(n) + ln) * RS + 4 * qd];
                const float* xrow = &sm.x[(16 * tile32_it(n) + ln) * RS + 4 * qd];
#pragma unroll
                for (int s = 0; s < D / 16; ++s) {
                    const f32x4 a = *reinterpret_cast<const f32x4*>(yrow + 16 * s);
                    const f32x4 b = *reinterpret_cast<const f32x4*>(xrow + 16 * s);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], acc, 0, 0, 0);
                }
                sm.pfrag[n][l] = acc * wgt[n / NW];
            }

            // O^T = S^T X^T, rows of O scaled by Lam
#pragma unroll
            for (int it = 0; it < 4; ++it) {
                f32x4 acc = {0.f, 0.f, 0.f, 0.f};
                const float* xrow = &sm.x[(16 * it + ln) * RS + 4 * qd];
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    const f32x4 b = *reinterpret_cast<const f32x4*>(xrow + 16 * dt);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(S[dt][e], b[e], acc, 0, 0, 0);
                }
                o[it] = acc * sm.pw[max(16 * it + ln + later - shift, 0)];
            }
        }

        // z registers: za[4jt + r] = Z[j = 16jt + 4q + r][c_own]
        float za[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) za[e] = sm.z[(16 * (e >> 2) + 4 * qd + (e & 3)) * RS + c_own];

        if (kOut) {
            __syncthreads();  // score fragments visible
            // O^T += Z^T P^T over the tiles (jt <= it)
#pragma unroll
            for (int n = 0; n < 10; ++n) {
                const f32x4 pt = sm.pfrag[n][l];
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    o[tile32_it(n)] = __builtin_amdgcn_mfma_f32_16x16x4f32(za[4 * tile32_jt(n) + r], pt[r], o[tile32_it(n)], 0, 0, 0);
            }
            // O^T: lane = token 16it + ln, registers = columns 16w + 4q + (0..3)
#pragma unroll
            for (int it = 0; it < 4; ++it) {
                const int i = 16 * it + ln;
                if (i >= shift)
                    __builtin_nontemporal_store(o[it], reinterpret_cast<f32x4*>(ob + (tok0 - shift + i) * row + 16 * w + 4 * qd));
            }
        }

        // S = gamma^L S + Y^T (Gam Z); contraction slot q of step (jt, r) is token 16jt + 4q + r
        const float gl = sm.pw[Lc];
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) S[dt] *= gl;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const float b = za[e] * gam[e];
            const float* yrow = &sm.y[(16 * (e >> 2) + 4 * qd + (e & 3)) * RS + ln];
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) S[dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(yrow[16 * dt], b, S[dt], 0, 0, 0);
        }
    }

    float* dst = nullptr;
    if (!kOut) dst = role.slots + ((size_t)bh * (p.nseg - 1) + seg) * D * D;
    else if (seg == p.nseg - 1 && role.leave) dst = role.leave + (size_t)bh * D * D;
    if (dst) {
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) dst[(16 * t + 4 * qd + r) * D + c_own] = S[t][r];
    }
}

template <bool kOut>
static hipError_t launch_width32(const BwdParams& p, int D, hipStream_t stream) {
    const int units = p.BH * (kOut ? p.nseg : p.nseg - 1);
    const dim3 grid((units + 7) / 8 * 8 * p.roles), block(D * 4);
    if (D == 64) hipLaunchKernelGGL((walk32_kernel<64, kOut>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((walk32_kernel<128, kOut>), grid, block, 0, stream, p);
    return hipGetLastError();
}

}  // namespace bwd

hipError_t launch_bwd_f32_states(const BwdParams& p, int D, hipStream_t stream) { return bwd::launch_width32<false>(p, D, stream); }
hipError_t launch_bwd_f32_walk(const BwdParams& p, int D, hipStream_t stream) { return bwd::launch_width32<true>(p, D, stream); }

}  // namespace leet
