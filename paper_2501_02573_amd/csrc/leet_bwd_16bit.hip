// Backward pass of the decayed causal linear attention for 16-bit inputs, bf16 or fp16 (gfx950,
// v_mfma_f32_32x32x16_{bf16,f16}, fp32 accumulate).
//
// With M[i][j] = gamma^(i-j) for i >= j (Section 2.2, Eq. "BCMV"; the paper has no backward pass) and dO the gradient of O:
//
//     dQ = ((dO V^T) .* M) K + (state)      dK = ((V dO^T) .* M^T) Q + (state)      dV = ((K Q^T) .* M^T) dO + (state)
//
// Each is the attention itself over other operands, out = ((X Y^T) .* M) Z: dQ in the order of the tokens with
// (X, Y, Z) = (dO, V, K), dK and dV in the reversed order, where M^T is M, with (V, dO, Q) and (K, Q, dO).  So one
// kernel walks the 64-token chunks of a segment in the role's order with the state S = sum of Y^T Z in MFMA accumulators,
// and the scores are formed again, never stored:
//
//     O_t     = ((X_t Y_t^T) .* D) Z_t + Lam (X_t S_t)       D[i][j] = gamma^(i-j), i >= j
//     S_{t+1} = gamma^L S_t + (Gam Y_t)^T Z_t
//
// In the order of the tokens S is the transposed state before a chunk: Lam = gamma^(i+1), Gam = gamma^(L-1-j).  Reversed, S
// is the gradient of the state that the chunk's last token leaves: Lam = gamma^i, Gam = gamma^(L-j).
//
// The three walks ask for nine tensors' worth (dout three times, v, q and k twice each) and read 6.8 to 7.3, as dK and dV, side by
// side on an XCD, meet in its L2; they write three.  Two kernels: walk16_kernel, many small workgroups, for any number of segments; and
// tiles16_kernel, one large workgroup a sequence, where there are few sequences.  With segments a pre-pass over the states
// of both directions (walk16_kernel without outputs) and the scan of their boundaries come first.
// Near memory's rate where the device is full: B16 H32 N2048 d128 bf16 takes 582 us, ten tensors at 4.6 TB/s (with one term 530,
// 5.1).  Few sequences are bound by a chunk's latency, or by segments' pre-pass, which reads four tensors again.  B4 H16 N4096: 174
// to 181 us in a run of calls (190 to 220 on a device that was idle), of which its 9.8 tensors are 128 at 5.1 TB/s; with dstate_in
// wanted and three terms 207 to 217.
#include <type_traits>

#include "leet_backward.hpp"
#include "leet_common.hpp"

namespace leet {
namespace bwd {

typedef short s16x4 __attribute__((ext_vector_type(4)));

template <int D, int DV>
struct Smem16 {
    static constexpr int RS = D + 8;                      // row strides (elements): 16-byte reads of 32 rows spread over the banks
    static constexpr int RSZ = DV + (DV > 128 ? 32 : 16);  // read through ds_read_b64_tr_b16 only; holds the output scratch
    uint16_t x[kChunk * RS];
    uint16_t y[kChunk * RS];
    uint16_t z[kChunk * RSZ];
    u32x4 pfrag[3][2][64];   // masked score tiles as B operands: [tile][register half][lane]
    float pw[kChunk + 4];    // gamma^n, n = 0..64
    float gw[kChunk];        // Gam
    float back[3][32];       // fp16: what undoes the scaling of a score tile's tokens
    float gw_held[DV / 32][kChunk];  // fp16: Gam times a wave's scale of z
};

// fp16's normal numbers reach from 2^-14 to 65504, fp32's values that become its operands lie anywhere: gradients of 2^-18 lost most
// of their bits below, scores and states of large ones became infinite where every gradient is finite.  So fp16 has powers of two:
//   * scores are brought to [2^14, 2^15) for each token of a tile as they become operands, and the product back;
//   * a state is kept times `held`, which Gam carries: the largest z of a chunk is brought to [2^8, 2^9), in three terms to [2^14,
//     2^15), and without decay z is taken 256 times where that is finite; where the largest of a wave's state then lies outside [4, 2^15) the state itself is brought to [2^14, 2^15).
// A rounding to one term is 2^-11 of the value, or 2^-25 of a number of that scale: 2^-39 of a token's largest score, 2^-27 of the
// largest of a state; what is added to a state is off by 2^-33 of the largest z (three terms 2^-39) or 2^-22 of itself (2^-24); without decay by nothing.
// The matrix instructions add products of numbers below 2^-14 as if these had that exponent.
// fp16 takes 6 to 18 % longer by it (a compute unit a sequence without decay 22 %).  us before and after: B16 H32 N2048 d128 594 642,
// B4 H16 N4096 d128 178 210 (without decay 149 182), B2 H16 130 137, B4 H16 N4096 d64 96.5 103.6, B3 H12 N1777 d64 34.5 37.5, B16 H32
// N128 d64 25.7 29.7, B2 H16 N2048 128/256 150 160.  (Scaling each state as it becomes an operand, and each column of z by itself:
// 223 instead of 210.)
template <typename E>
constexpr bool kNarrow = std::is_same<E, ElemF16>::value;

// m >= 0: the power of two that brings values of up to m, 2^kLeast at least, to [2^kTo, 2^(kTo + 1)).  Infinities stay infinite.
template <int kTo, int kLeast>
__device__ __forceinline__ float power_to(float m) {
    return __uint_as_float(((254u + kTo) << 23) - max(__float_as_uint(m) & 0x7f800000u, (127u + kLeast) << 23));
}
// 1 / x of a power of two
__device__ __forceinline__ float inverse_of(float x) { return __uint_as_float((254u << 23) - __float_as_uint(x)); }
// Smaller scores are not brought up further, so that sums of them with what is not small (times 2^60) stay finite: rounded to 2^-85
// they add 2^-63 to an output at most, whose least number is 2^-24.
__device__ __forceinline__ float power_of_scores(float m) { return power_to<14, -46>(m); }

__device__ __forceinline__ float most_of(const f32x16& v, float m) {
#pragma unroll
    for (int r = 0; r < 16; ++r) m = fmaxf(m, fabsf(v[r]));
    return m;
}
// The larger one of lanes l and l ^ 32; numbers >= 0 as their bits, of which NaNs are the largest.
__device__ __forceinline__ uint32_t most_of_halves(uint32_t m) {
    const u32x2 both = __builtin_amdgcn_permlane32_swap(m, m, false, false);
    return max(both[0], both[1]);
}
template <int kCtrl>
__device__ __forceinline__ uint32_t most_dpp(uint32_t m) {
    return max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, kCtrl, 0xf, 0xf, true));
}
// the largest of a wave's lanes, the same in all of them
__device__ __forceinline__ uint32_t most_of_wave(uint32_t m) {
    m = most_dpp<0xB1>(m);   // quad_perm 1 0 3 2
    m = most_dpp<0x4E>(m);   // quad_perm 2 3 0 1
    m = most_dpp<0x141>(m);  // row_half_mirror
    m = most_dpp<0x140>(m);  // row_mirror
    const u32x2 both = __builtin_amdgcn_permlane16_swap(m, m, false, false);
    return __builtin_amdgcn_readfirstlane(most_of_halves(max(both[0], both[1])));
}
// of a score tile's column, a token
__device__ __forceinline__ float most_of_token(const f32x16& v) {
    return __uint_as_float(most_of_halves(__float_as_uint(most_of(v, 0.0f))));
}
// of all lanes but those that are infinite or NaN: finite columns of a state keep their bits beside others
__device__ __forceinline__ float most_finite(float m) {
    return __uint_as_float(most_of_wave(m < __builtin_inff() ? __float_as_uint(m) : 0u));
}
// The largest finite one of a wave's fp16 values; kColumns: a lane's values are of one column, which is lost where one of them is
// infinite or NaN, and are left out then.
template <bool kColumns, int kCount>
__device__ __forceinline__ float most_of_rows(const u32x4 (&v)[kCount]) {
    typedef _Float16 Pair __attribute__((ext_vector_type(2)));
    typedef uint16_t Bits __attribute__((ext_vector_type(2)));
    Pair high = {0, 0}, low = {0, 0};
#pragma unroll
    for (int f = 0; f < kCount; ++f)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t word = v[f][e];
            high = __builtin_elementwise_maximum(high, __builtin_bit_cast(Pair, word));
            low = __builtin_elementwise_minimum(low, __builtin_bit_cast(Pair, word));
        }
    Bits most = __builtin_bit_cast(Bits, __builtin_elementwise_maximum(high, -low));
    uint32_t m = max(most[0], most[1]);
    if (kColumns) {
        m = m < 0x7c00u ? m : 0u;
    } else if (__builtin_expect(m >= 0x7c00u, 0)) {  // 2^10 more than their bits wraps to less than any finite number's
        most = Bits{0, 0};
#pragma unroll
        for (int f = 0; f < kCount; ++f)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t word = v[f][e];
                most = __builtin_elementwise_max(most, (__builtin_bit_cast(Bits, word) + (uint16_t)0x400) & (uint16_t)0x7fff);
            }
        m = max((uint32_t)max(most[0], most[1]), 0x400u) - 0x400u;
    }
    return (float)__builtin_bit_cast(_Float16, (uint16_t)most_of_wave(m));
}
// The scale of z in a chunk, no more than leaves a state of up to 2^15 / held finite.  Without decay (kTerms 1) it is 2^8 or 1, which
// lose no bit, and mostly the last chunk's.
template <int kTerms>
__device__ __forceinline__ float power_of_z(float most, float held) {
    const float by = kTerms == 1 ? (most < 128.0f ? 256.0f : 1.0f) : power_to<kTerms == 2 ? 8 : 14, -24>(most);
    return fminf(by, 0x1p85f * held);
}
// Brings a wave's state, of which it holds `held` times, into fp16's range.
template <int kTiles>
__device__ __forceinline__ void keep_in_range(f32x16 (&S)[kTiles], float& held) {
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < kTiles; ++i) m = most_of(S[i], m);
    m = most_finite(m);
    if (m >= 0x1p15f || (m < 4.0f && m > 0.0f)) {  // the same in all lanes
        const float by = fminf(power_to<14, -99>(m), 0x1p100f * inverse_of(held));  // so that `held` stays finite
        held *= by;
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) S[i][r] *= by;
    }
}

__device__ __forceinline__ u32x4 frag16(const uint16_t* p) { return *reinterpret_cast<const u32x4*>(p); }

// ds_read_b64_tr_b16: within each group of 16 lanes, lane i receives element i%4 of the 8-byte rows addressed by lanes
// i/4, 4+i/4, 8+i/4, 12+i/4 of the group.
__device__ __forceinline__ u32x2 lds_tr(const uint16_t* p) {
    s16x4 r = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) s16x4*)(const_cast<uint16_t*>(p)));
    return __builtin_bit_cast(u32x2, r);
}
__device__ __forceinline__ u32x4 join(u32x2 a, u32x2 b) { return u32x4{a.x, a.y, b.x, b.y}; }

// registers 8h .. 8h+7 of an accumulator tile -> 16-bit operand
template <typename E>
__device__ __forceinline__ u32x4 pack_half(const f32x16& acc, int h) {
    u32x4 r;
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = E::pack2(acc[8 * h + 2 * e], acc[8 * h + 2 * e + 1]);
    return r;
}

// what pack_half rounded off, as a 16-bit operand of its own
template <typename E>
__device__ __forceinline__ u32x4 pack_rest(const f32x16& acc, u32x4 packed, int h) {
    u32x4 r;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        r[e] = E::pack2(acc[8 * h + 2 * e] - E::lo(packed[e]), acc[8 * h + 2 * e + 1] - E::hi(packed[e]));
    return r;
}

// Eight 16-bit values times eight fp32 weights as kTerms 16-bit values that add up to the product.  What is left for the next
// term is taken from the packed word itself: the compiler may form the fp16 of a product in two ways, once from the product
// rounded to fp32 and once not, and the two differ now and then by a step.
template <typename E, int kTerms>
__device__ __forceinline__ void scaled(u32x4 x, f32x4 w0, f32x4 w1, u32x4 (&out)[kTerms]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float a = E::lo(x[e]) * ((e < 2) ? w0[2 * e] : w1[2 * e - 4]);
        float b = E::hi(x[e]) * ((e < 2) ? w0[2 * e + 1] : w1[2 * e - 3]);
#pragma unroll
        for (int t = 0; t < kTerms; ++t) {
            uint32_t word = E::pack2(a, b);
            if (t + 1 < kTerms) asm("" : "+v"(word));
            out[t][e] = word;
            a -= E::lo(word);
            b -= E::hi(word);
        }
    }
}

// eight fp16 values times a power of two
__device__ __forceinline__ u32x4 times_power(u32x4 x, float by) {
    const f16x8 v = __builtin_bit_cast(f16x8, x) * (_Float16)by;
    return __builtin_bit_cast(u32x4, v);
}

// The rows of a sequence that hold tokens tok0 .. tok0 + L - 1 of a walk (rows of `width` elements; `seq`: its first row), L = 64
// or what is left of its N, as a buffer: what lies outside it is read as zero and not written, so that loads and stores
// need no branches, behind which the compiler could no longer count those under way.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t chunk_rows(const void* seq, int width, bool rev, int N, int tok0) {
    const int L = max(min(kChunk, N - tok0), 0);
    const uintptr_t addr = reinterpret_cast<uintptr_t>(seq) + (size_t)(rev ? N - tok0 - L : tok0) * (width * 2);
    // the same in every lane; the compiler is told
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)addr), hi = __builtin_amdgcn_readfirstlane((uint32_t)(addr >> 32));
    return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(((uintptr_t)hi << 32) | lo), 0,
                                             __builtin_amdgcn_readfirstlane(L * width * 2), 0x00027000);
}
// Where row i of a chunk's tile begins in there.  A ragged chunk is right-aligned in the tile: rows above its first one, `shift`,
// lie outside.
__device__ __forceinline__ int row_at(int i, int width, bool rev, int shift) { return (rev ? kChunk - 1 - i : i - shift) * (width * 2); }

// Score tiles in production order: tile 0 = (jt 0, it 0), tile 1 = (jt 1, it 1), tile 2 = (jt 0, it 1).
__device__ __forceinline__ constexpr int tile_jt(int n) { return n == 1 ? 1 : 0; }
__device__ __forceinline__ constexpr int tile_it(int n) { return n == 0 ? 0 : 1; }

// kOut = true: outputs and state.  kOut = false: state only, of every segment but the last, started from zero.
// kTerms: of Gam Z, whose rounding to one would be as large as the outputs' own (two: the outputs' error falls from 1.65 to 1.4
// times that of outputs that are rounded alone; B4 H16 N4096 d128 bf16 155 -> 173 us).  Three give a leaving state to fp32's
// precision.
// kFew: scores and states, rounded to 16 bits as operands elsewhere, are taken in two terms; sequences of one or two chunks.  Over
// a few tokens their errors do not average out (an output is one or two products), and one token's gradients were off by up to
// 2.5 times what outputs that are rounded alone are.  From 128 tokens on one term makes it 1.42 to 1.45 times.  Takes 12 to 18 %
// longer (B16 H32 N128 bf16: d 64 18.8 -> 22.1 us, d 128 38.0 -> 44.2).
template <int D, int DV, bool kOut, typename E, bool kDecay, int kTerms, bool kFew>
__global__ __launch_bounds__(DV * 2, D > 128 || DV > 128 ? 1 : 2) void walk16_kernel(BwdParams p) {
    constexpr int NT = DV * 2;   // threads: one wave per 32 columns of z and out
    constexpr int NW = DV / 32;  // waves
    constexpr int DT = D / 32;   // 32-row tiles of the state
    constexpr int PR = D / 8, PRZ = DV / 8;  // 16-byte pieces per row
    constexpr int XP = kChunk * PR / NT, ZP = kChunk * PRZ / NT;  // pieces per thread per chunk
    constexpr int RS = Smem16<D, DV>::RS, RSZ = Smem16<D, DV>::RSZ;
    static_assert(kChunk * RSZ * 2 >= NW * 32 * 20 * 4, "the z tile must hold the output scratch");
    __shared__ __attribute__((aligned(16))) Smem16<D, DV> sm;

    const int tid = threadIdx.x;
    const int w = tid >> 6, l = tid & 63, ln = l & 31, g = l >> 5;
    // workgroups go to the eight XCDs in turn: the roles of a unit share an XCD's L2
    const int nseg = kOut ? p.nseg : p.nseg - 1;
    const int slot = blockIdx.x >> 3, which = slot % p.roles, unit = (slot / p.roles) * 8 + (blockIdx.x & 7);
    if (unit >= p.BH * nseg) return;
    const BwdRole& role = p.role[which];
    const bool rev = role.reversed != 0;
    const int bh = unit / nseg;
    const int seg = rev ? nseg - 1 - unit % nseg : unit % nseg;
    const int h = bh % p.H;

    const int tok_begin = seg * p.seg_chunks * kChunk;
    const int tok_end = (seg == p.nseg - 1) ? p.N : tok_begin + p.seg_chunks * kChunk;
    const int nchunks = (tok_end - tok_begin + kChunk - 1) / kChunk;

    // token t of the walk is row t, or N - 1 - t, of the tensors
    const size_t first = (size_t)bh * p.N + (rev ? p.N - 1 : 0);
    const ptrdiff_t row = rev ? -D : D, row_z = rev ? -DV : DV;
    const uint16_t* xb = static_cast<const uint16_t*>(role.x) + first * D;
    const uint16_t* yb = static_cast<const uint16_t*>(role.y) + first * D;
    const uint16_t* zb = static_cast<const uint16_t*>(role.z) + first * DV;
    uint16_t* ob = static_cast<uint16_t*>(role.out) + first * DV;

    if (kDecay) {  // fp64 -> fp32 once per workgroup
        const double gd = (double)p.gamma[h];
        for (int n = tid; n <= kChunk; n += NT) {
            const float v = (float)pow_int(gd, n);
            sm.pw[n] = v;
            const int j = kChunk - 1 + (rev ? 1 : 0) - n;
            if (j >= 0 && j < kChunk) sm.gw[j] = v;
        }
    }

    // state slice: S[t][r] = S[dk = 32t + pi(m(r, g))][c = 32w + ln]; in fp16 times `held`
    f32x16 S[DT];
    float held = 1.0f;  // the same in all lanes
    const int c_own = 32 * w + ln;
    auto dk_of = [&](int t, int r) {
        // m = 8(r/4) + 4g + r%4 ; pi swaps the 4- and 8-bits: dk = 16(r/8) + 8g + 4((r/4)&1) + r%4
        return 32 * t + 16 * (r >> 3) + 8 * g + 4 * ((r >> 2) & 1) + (r & 3);
    };
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) S[t][r] = 0.0f;
    if (kOut && seg > 0) {
        const float* src = role.slots + ((size_t)bh * (p.nseg - 1) + seg - 1) * D * DV + (size_t)c_own * role.slot_col;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) S[t][r] = src[dk_of(t, r) * role.slot_row];
    }
    if (kOut && role.enter) {
        const float* src = role.enter + (size_t)bh * D * DV + (size_t)c_own * role.enter_col;
        const float left = kDecay ? (float)pow_int((double)p.gamma[h], tok_begin) : 1.0f;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) S[t][r] += left * src[dk_of(t, r) * role.enter_row];
    }

    // per-lane LDS bases; every fragment address below is one of these plus a constant
    const int s16 = l & 15, half = (l >> 4) & 1;
    const uint16_t* x_row = &sm.x[ln * RS + 8 * g];   // + 32*it*RS + 16*s
    const uint16_t* y_row = &sm.y[ln * RS + 8 * g];   // + 32*jt*RS + 16*s
    // transposing reads: lane supplies row 4g + s16/4 (+ 8*rd + 16*f) and four consecutive columns
    const uint16_t* z_tr = &sm.z[(4 * g + (s16 >> 2)) * RSZ + 32 * w + 16 * half + 4 * (s16 & 3)];
    const uint16_t* y_tr = &sm.y[(4 * g + (s16 >> 2)) * RS + 16 * half + 8 * (s16 & 1) + 4 * ((s16 >> 1) & 1)];
    float* gw = kNarrow<E> ? sm.gw_held[w] : sm.gw;

    __syncthreads();  // tables visible

    // Decay weights of the score tiles this wave produces.  wgt[0]: a tile on the diagonal (i - j = ln - jr, zero above the
    // diagonal); wgt[1]: the tile below it (i - j = 32 + ln - jr).  With four waves each wave needs one set.
    constexpr bool kBothSets = NW < 3;
    f32x16 wgt[kBothSets ? 2 : 1];
    const int later = rev ? 0 : 1;
    float lam_full[2];  // Lam of a full chunk
    if (kOut) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int n = ln - (8 * (r >> 2) + 4 * g + (r & 3));
            const float diag = (n >= 0) ? (kDecay ? sm.pw[max(n, 0)] : 1.0f) : 0.0f;
            const float below = kDecay ? sm.pw[32 + n] : 1.0f;
            if (kBothSets) {
                wgt[0][r] = diag;
                wgt[kBothSets ? 1 : 0][r] = below;
            } else {
                wgt[0][r] = (w == 2) ? below : diag;
            }
        }
        lam_full[0] = kDecay ? sm.pw[ln + later] : 1.0f;
        lam_full[1] = kDecay ? sm.pw[32 + ln + later] : 1.0f;
    }

    u32x4 rx[XP], ry[XP], rz[ZP];
    auto prefetch = [&](int tok0) {
        const int shift = max(0, tok0 + kChunk - tok_end);  // rows [0, shift) of the tile stay zero
        const u32x4 zero = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int r = 0; r < XP; ++r) {
            const int piece = r * NT + tid, j = piece / PR, cc = piece % PR;
            const bool ok = j >= shift;
            const ptrdiff_t off = (tok0 - shift + j) * row + cc * 8;
            if (kOut) rx[r] = ok ? *reinterpret_cast<const u32x4*>(xb + off) : zero;
            ry[r] = ok ? *reinterpret_cast<const u32x4*>(yb + off) : zero;
        }
#pragma unroll
        for (int r = 0; r < ZP; ++r) {
            const int piece = r * NT + tid, j = piece / PRZ, cc = piece % PRZ;
            const ptrdiff_t off = (tok0 - shift + j) * row_z + cc * 8;
            rz[r] = j >= shift ? *reinterpret_cast<const u32x4*>(zb + off) : zero;
        }
    };

    prefetch(tok_begin);

    for (int t = 0; t < nchunks; ++t) {
        const int tok0 = tok_begin + t * kChunk;
        const int Lc = min(kChunk, tok_end - tok0);
        const int shift = kChunk - Lc;  // a ragged last chunk is right-aligned in the tile, rows above are zero

        if (t > 0) __syncthreads();  // everyone is done reading the previous chunk's tiles and score fragments
#pragma unroll
        for (int r = 0; r < XP; ++r) {
            const int piece = r * NT + tid, j = piece / PR, cc = piece % PR;
            if (kOut) *reinterpret_cast<u32x4*>(&sm.x[j * RS + cc * 8]) = rx[r];
            *reinterpret_cast<u32x4*>(&sm.y[j * RS + cc * 8]) = ry[r];
        }
#pragma unroll
        for (int r = 0; r < ZP; ++r) {
            const int piece = r * NT + tid, j = piece / PRZ, cc = piece % PRZ;
            *reinterpret_cast<u32x4*>(&sm.z[j * RSZ + cc * 8]) = rz[r];
        }
        __syncthreads();
        if (t + 1 < nchunks) prefetch(tok0 + kChunk);  // in flight during the MFMA work below

        f32x16 o[2];
        float lam[2];
        u32x4 rest[kFew ? (3 + NW - 1) / NW : 1][2];
        if (kOut) {
            // P^T = Y X^T, masked, for the score tiles this wave produces
#pragma unroll
            for (int n = 0; n < 3; ++n) {
                if (n % NW != w) continue;
                f32x16 acc;
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[r] = 0.0f;
#pragma unroll
                for (int s = 0; s < D / 16; ++s)
                    acc = E::mfma32(frag16(y_row + 32 * tile_jt(n) * RS + 16 * s),
                                    frag16(x_row + 32 * tile_it(n) * RS + 16 * s), acc);
                if (kDecay || n != 2) {  // without decay the tile below the diagonal needs no weights
                    const f32x16& wt = wgt[(kBothSets && n == 2) ? 1 : 0];
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[r] *= wt[r];
                }
                if (kNarrow<E>) {
                    const float up = power_of_scores(most_of_token(acc));
                    sm.back[n][ln] = inverse_of(up);
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[r] *= up;
                }
#pragma unroll
                for (int hh = 0; hh < 2; ++hh) {
                    const u32x4 packed = pack_half<E>(acc, hh);
                    sm.pfrag[n][hh][l] = packed;
                    if (kFew) rest[n / NW][hh] = pack_rest<E>(acc, packed, hh);
                }
            }

            // O^T = S^T X^T, rows of O scaled by Lam
            lam[0] = lam_full[0];
            lam[1] = lam_full[1];
            if (kDecay && shift) {
                lam[0] = sm.pw[max(ln + later - shift, 0)];
                lam[1] = sm.pw[max(32 + ln + later - shift, 0)];
            }
#pragma unroll
            for (int it = 0; it < 2; ++it)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[it][r] = 0.0f;
            if constexpr (kNarrow<E>) {
                keep_in_range(S, held);
                lam[0] *= inverse_of(held);
                lam[1] *= inverse_of(held);
            }
#pragma unroll
            for (int s = 0; s < D / 16; ++s) {
                const u32x4 sa = pack_half<E>(S[s >> 1], s & 1);
                const u32x4 sb = kFew ? pack_rest<E>(S[s >> 1], sa, s & 1) : sa;
#pragma unroll
                for (int it = 0; it < 2; ++it) {
                    const u32x4 xf = frag16(x_row + 32 * it * RS + 16 * s);
                    o[it] = E::mfma32(sa, xf, o[it]);
                    if (kFew) o[it] = E::mfma32(sb, xf, o[it]);
                }
            }
            if (kDecay && !kNarrow<E>) {
#pragma unroll
                for (int it = 0; it < 2; ++it)
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[it][r] *= lam[it];
            }
        }

        // z fragments: zf[f], f = 2*jt + hh, holds tokens 16f + {4g..4g+3, 8+4g..8+4g+3} of column c_own
        u32x4 zf[4];
#pragma unroll
        for (int f = 0; f < 4; ++f) zf[f] = join(lds_tr(z_tr + (16 * f) * RSZ), lds_tr(z_tr + (16 * f + 8) * RSZ));

        if (kOut) {
            __syncthreads();  // score fragments visible; the z tile is dead: its fragments are in registers
            // O^T += Z^T P^T over the tiles (jt <= it)
            // (fp16: the sums are brought to a tile's scale before it and, behind the last, back)
            auto add_tiles = [&](float first0, float first1) {
                float to[2] = {first0, first1};
#pragma unroll
                for (int n = 0; n < 3; ++n) {
                    f32x16& sum = o[tile_it(n)];
                    if (kNarrow<E>) {
                        const float down = sm.back[n][ln];
                        // (sums that this limit leaves too small are far beyond 65504 all the same; it keeps zeros from becoming NaN)
                        const float by = fminf(to[tile_it(n)] * inverse_of(down), 0x1p127f);
                        to[tile_it(n)] = down;
#pragma unroll
                        for (int r = 0; r < 16; ++r) sum[r] *= by;
                    }
#pragma unroll
                    for (int hh = 0; hh < 2; ++hh) sum = E::mfma32(zf[2 * tile_jt(n) + hh], sm.pfrag[n][hh][l], sum);
                }
                if (kNarrow<E>) {
#pragma unroll
                    for (int it = 0; it < 2; ++it)
#pragma unroll
                        for (int r = 0; r < 16; ++r) o[it][r] *= to[it];
                }
            };
            add_tiles(lam[0], lam[1]);
            if (kFew) {  // the same with what the scores were rounded by
                __syncthreads();
#pragma unroll
                for (int n = 0; n < 3; ++n) {
                    if (n % NW != w) continue;
#pragma unroll
                    for (int hh = 0; hh < 2; ++hh) sm.pfrag[n][hh][l] = rest[n / NW][hh];
                }
                __syncthreads();
                add_tiles(1.0f, 1.0f);
            }

            // O^T: lane = token 32it + ln, registers 4q..4q+3 = columns 32w + 8q + 4g + (0..3).  Through a wave-private LDS
            // tile so that a store covers whole 64-byte row pieces: lane -> (row l/4, 16 bytes l%4).
            uint32_t* scr = reinterpret_cast<uint32_t*>(sm.z) + w * (32 * 20);
#pragma unroll
            for (int it = 0; it < 2; ++it) {
#pragma unroll
                for (int qd = 0; qd < 4; ++qd) {
                    const u32x2 val = {E::pack2(o[it][4 * qd], o[it][4 * qd + 1]), E::pack2(o[it][4 * qd + 2], o[it][4 * qd + 3])};
                    *reinterpret_cast<u32x2*>(scr + ln * 20 + 4 * qd + 2 * g) = val;
                }
                u32x4 val[2];
#pragma unroll
                for (int m = 0; m < 2; ++m) val[m] = *reinterpret_cast<const u32x4*>(scr + (16 * m + (l >> 2)) * 20 + 4 * (l & 3));
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    const int i = 32 * it + 16 * m + (l >> 2);
                    if (i >= shift)
                        __builtin_nontemporal_store(val[m], reinterpret_cast<u32x4*>(ob + (tok0 - shift + i) * row_z + 32 * w + 8 * (l & 3)));
                }
            }
        }

        // S = gamma^L S + Y^T (Gam Z)
        if (kDecay || kNarrow<E>) {
            float gl = kDecay ? sm.pw[Lc] : 1.0f;
            if constexpr (kNarrow<E>) {
                const float next = power_of_z<kTerms>(most_of_rows<true>(zf), kOut ? held : 1.0f);
                gl *= next * inverse_of(held);
                held = next;
                if (kDecay) gw[l] = sm.gw[l] * held;  // read by this wave alone
            }
            if (kDecay || gl != 1.0f) {  // the same in all lanes
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                    for (int r = 0; r < 16; ++r) S[dt][r] *= gl;
            }
        }
#pragma unroll
        for (int f = 0; f < 4; ++f) {
            u32x4 zs[kTerms];
            if (kDecay)
                scaled<E, kTerms>(zf[f], *reinterpret_cast<const f32x4*>(&gw[16 * f + 4 * g]),
                                  *reinterpret_cast<const f32x4*>(&gw[16 * f + 8 + 4 * g]), zs);
            else if (kNarrow<E>) zs[0] = times_power(zf[f], held);
            else zs[0] = zf[f];
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                const u32x4 a = join(lds_tr(y_tr + (16 * f) * RS + 32 * dt), lds_tr(y_tr + (16 * f + 8) * RS + 32 * dt));
#pragma unroll
                for (int u = 0; u < kTerms; ++u) S[dt] = E::mfma32(a, zs[u], S[dt]);
            }
        }
    }

    // hand the state on
    float* dst = nullptr;
    if (!kOut) dst = role.slots + ((size_t)bh * (p.nseg - 1) + seg) * D * DV;
    else if (seg == p.nseg - 1 && role.leave) dst = role.leave + (size_t)bh * D * DV;
    if (dst) {
        const float real = kNarrow<E> ? inverse_of(held) : 1.0f;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) dst[dk_of(t, r) * DV + c_own] = kNarrow<E> ? S[t][r] * real : S[t][r];
    }
}

// ---- both widths 128: a wave for each 32 x 32 tile of the outputs ----
//
// What bounds a walk that has a compute unit to itself is the time that one chunk takes after the other, so here twice as many
// waves share it, two a SIMD: wave (c, it) forms O^T[32 columns c][32 rows it] and carries the half `it` of the state's rows
// for its columns.  A chunk has two halves with a barrier behind each:
//   1  the next chunk's tiles into a second set of buffers; what comes from the state behind the last chunk, S^T X^T; the half
//      `it` of the columns' z rows times Gam, to LDS as the operands that they will be;
//   2  the state's update, and the new state to LDS as the 16-bit operand of the next chunk; Z^T P^T and the output; the next
//      chunk's three score tiles, one each in three waves, to LDS as operands.
// So what one half needs of another wave is formed in the half before it, and loads are under way for a chunk's time.
//
// A chunk of a role takes 2.3 us with a few workgroups on the device, the latency of its dependent steps (LDS operands and matrix
// instructions, two waves a SIMD); with 192, 2.7, where memory shows: B4 H16 N4096 bf16 alone reading 74 us, alone storing 58,
// both 137, alone computing 150, all 179.  Tried: four waves, three buffers and one barrier a chunk 184 to 205 us; loads two
// chunks ahead, no change; outputs held back and stored as whole rows through LDS 180.  Stores are cached: 32-byte pieces of
// rows that go past the cache take 1.8 times as long.
//
// A tile's rows are unpadded; 16-byte piece p of row r sits at piece p ^ turn(r).  Reads of one piece of 16 rows (operands
// along a row) and transposing reads of four rows and four pieces meet every bank once.
__device__ __forceinline__ constexpr int turn(int row) { return 4 * (row & 3) + ((row >> 2) & 3); }

struct SmemTiles {
    static constexpr int D = 128;
    uint16_t x[2][kChunk * D], y[2][kChunk * D], z[2][kChunk * D];
    uint16_t st[D * D];               // S^T[c][dk], turned as the tiles are
    u32x4 pfrag[2][3][2][64];         // masked score tiles as B operands: [buffer][tile][register half][lane]
    u32x4 zfrag[D / 32][4][64];       // Gam Z as B operands: [column tile][16 tokens][lane]
    float pw[kChunk + 4];             // gamma^n, n = 0..64
    float gw[kChunk];                 // Gam
};
// fp16 has also
struct SmemScales {
    float back[2][3][32];             // what undoes the scaling of a score tile's tokens
    float st_back[2][2][4];           // and of a wave's state; two, as `scale` reads the one before the last chunk
    float z_most[2][8];               // a chunk's largest z, by wave
    float gw[2][kChunk];              // Gam times the scale of the chunk's z
    float held[2];                    // that scale
};

template <typename E, bool kDecay, int kTerms>
__global__ __launch_bounds__(SmemTiles::D * 4, 2) void tiles16_kernel(BwdParams p) {
    constexpr int D = SmemTiles::D;
    constexpr int NT = D * 4;         // threads
    constexpr int CT = D / 32;        // column tiles
    constexpr int HT = D / 64;        // 32-row tiles of the state that a wave carries
    constexpr int PR = D / 8;         // 16-byte pieces per row
    constexpr int LP = kChunk * PR / NT;  // pieces per thread per tensor per chunk (= 2)
    constexpr int LR = NT / PR;           // rows apart (= 32)
    __shared__ __attribute__((aligned(16))) SmemTiles sm;
    __shared__ __attribute__((aligned(16))) typename std::conditional<kNarrow<E>, SmemScales, int>::type scales;

    const int tid = threadIdx.x;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6), l = tid & 63, ln = l & 31, g = l >> 5;
    const int c = w % CT, it = w / CT;
    const int slot = blockIdx.x >> 3, which = slot % p.roles, unit = (slot / p.roles) * 8 + (blockIdx.x & 7);
    if (unit >= p.BH) return;
    const BwdRole& role = p.role[which];
    const bool rev = role.reversed != 0;
    const int nchunks = (p.N + kChunk - 1) / kChunk;

    // token t of the walk is row t, or N - 1 - t, of the sequence
    const size_t seq = (size_t)unit * p.N * D;
    const uint16_t *xb = static_cast<const uint16_t*>(role.x) + seq, *yb = static_cast<const uint16_t*>(role.y) + seq;
    const uint16_t* zb = static_cast<const uint16_t*>(role.z) + seq;
    uint16_t* ob = static_cast<uint16_t*>(role.out) + seq;

    // the chunk ahead, in registers
    struct Ahead {
        u32x4 x[LP], y[LP], z[LP];
    } ahead;
    const int j_own = tid / PR, cc = tid % PR;
    auto fetch = [&](int t) {  // zeros behind the last chunk
        const int tok0 = t * kChunk, shift = max(0, tok0 + kChunk - p.N);
        const auto xr = chunk_rows(xb, D, rev, p.N, tok0), yr = chunk_rows(yb, D, rev, p.N, tok0);
        const auto zr = chunk_rows(zb, D, rev, p.N, tok0);
#pragma unroll
        for (int r = 0; r < LP; ++r) {
            const int off = row_at(r * LR + j_own, D, rev, shift) + cc * 16;
            ahead.x[r] = __builtin_amdgcn_raw_buffer_load_b128(xr, off, 0, 0);
            ahead.y[r] = __builtin_amdgcn_raw_buffer_load_b128(yr, off, 0, 0);
            ahead.z[r] = __builtin_amdgcn_raw_buffer_load_b128(zr, off, 0, 0);
        }
    };
    const int to_own = (j_own * PR + (cc ^ turn(j_own))) * 8;
    auto put = [&](const Ahead& a, int buf) {
#pragma unroll
        for (int r = 0; r < LP; ++r) {
            *reinterpret_cast<u32x4*>(&sm.x[buf][to_own + r * LR * D]) = a.x[r];
            *reinterpret_cast<u32x4*>(&sm.y[buf][to_own + r * LR * D]) = a.y[r];
            *reinterpret_cast<u32x4*>(&sm.z[buf][to_own + r * LR * D]) = a.z[r];
        }
        if constexpr (kNarrow<E>) scales.z_most[buf][w] = most_of_rows<false>(a.z);
    };
    // fp16: what the chunk in buffer buf is scaled by, from its z and the states before the last chunk; a wave without a score tile
    auto scale = [&](int buf, int from) {
        if constexpr (kNarrow<E>) {
            if (w != 3) return;
            const f32x4 *z = reinterpret_cast<const f32x4*>(scales.z_most[buf]), *st = reinterpret_cast<const f32x4*>(scales.st_back[from]);
            float zm = 0.0f, back = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                zm = fmaxf(zm, z[i / 4][i % 4]);
                back = fmaxf(back, st[i / 4][i % 4]);
            }
            const float next = power_of_z<kTerms>(zm, inverse_of(back));
            scales.held[buf] = next;
            if (kDecay) scales.gw[buf][l] = sm.gw[l] * next;
        }
    };
    fetch(0);

    if (kDecay) {  // fp64 -> fp32 once per workgroup
        const double gd = (double)p.gamma[unit % p.H];
        for (int n = tid; n <= kChunk; n += NT) {
            const float v = (float)pow_int(gd, n);
            sm.pw[n] = v;
            const int j = kChunk - 1 + (rev ? 1 : 0) - n;
            if (j >= 0 && j < kChunk) sm.gw[j] = v;
        }
    }

    // state: S[i][r] = S[dk = 32 (HT it + i) + pi(m(r, g))][column 32c + ln]; in fp16 times `held`
    f32x16 S[HT];
    float held = 1.0f;  // the same in all lanes
    const int c_own = 32 * c + ln;
    auto dk_of = [&](int i, int r) { return 32 * (HT * it + i) + 16 * (r >> 3) + 8 * g + 4 * ((r >> 2) & 1) + (r & 3); };
#pragma unroll
    for (int i = 0; i < HT; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) S[i][r] = 0.0f;
    if (role.enter) {
        const float* src = role.enter + (size_t)unit * D * D + (size_t)c_own * role.enter_col;
#pragma unroll
        for (int i = 0; i < HT; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) S[i][r] = src[dk_of(i, r) * role.enter_row];
    }

    // Offsets (elements).  Operands along a row: piece 2s + g of row ln; the state's pieces of column ln likewise.
    int at_row[D / 16];
#pragma unroll
    for (int s = 0; s < D / 16; ++s) at_row[s] = ln * D + (((2 * s) ^ g ^ turn(ln)) * 8);
    // Transposing reads: row 4g + s16/4 (+ 8 rd + 16 f), four columns.  Eight rows on, a row's turn differs by 2.
    const int s16 = l & 15, half = (l >> 4) & 1, r_tr = 4 * g + (s16 >> 2);
    int z_tr[2], y_tr[HT][2];
#pragma unroll
    for (int rd = 0; rd < 2; ++rd) {
        const int t = turn(r_tr + 8 * rd), at = (r_tr + 8 * rd) * D;
        z_tr[rd] = at + ((4 * c + 2 * half + ((s16 >> 1) & 1)) ^ t) * 8 + 4 * (s16 & 1);
#pragma unroll
        for (int i = 0; i < HT; ++i) y_tr[i][rd] = at + ((4 * (HT * it + i) + 2 * half + (s16 & 1)) ^ t) * 8 + 4 * ((s16 >> 1) & 1);
    }
    auto gam_of = [&](int buf, int f, int more) {
        if constexpr (kNarrow<E>) return *reinterpret_cast<const f32x4*>(&scales.gw[buf][16 * f + 4 * g + more]);
        else return *reinterpret_cast<const f32x4*>(&sm.gw[16 * f + 4 * g + more]);
    };
    auto publish = [&](int buf) {
        if constexpr (kNarrow<E>) {
            keep_in_range(S, held);
            scales.st_back[buf][it][c] = inverse_of(held);
        }
#pragma unroll
        for (int i = 0; i < HT; ++i)
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) {
                // eight consecutive dk, piece 2 (2 tile + hh) + g of the column
                const int s2 = 2 * (2 * (HT * it + i) + hh);
                *reinterpret_cast<u32x4*>(&sm.st[32 * c * D + ln * D + ((s2 ^ g ^ turn(ln)) * 8)]) = pack_half<E>(S[i], hh);
            }
    };
    publish(0);
    put(ahead, 0);
    fetch(1);
    __syncthreads();  // tables and the first chunk visible

    // The score tile that this wave forms, if any: 0 = (jt 0, it 0), 1 = (1, 1), 2 = (0, 1), by waves of its rows on SIMDs of
    // their own.  Decay weights: on the diagonal i - j = ln - jr (zero above it), below it 32 + ln - jr.
    const int later = rev ? 0 : 1;
    const int tile = it == 0 ? (c == 0 ? 0 : -1) : c == 1 ? 1 : c == 2 ? 2 : -1;
    f32x16 wgt;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int n = ln - (8 * (r >> 2) + 4 * g + (r & 3)) + (tile == 2 ? 32 : 0);
        const float gn = kDecay ? sm.pw[max(n, 0)] : 1.0f;
        wgt[r] = n >= 0 ? gn : 0.0f;
    }
    const float lam_full = kDecay ? sm.pw[32 * it + ln + later] : 1.0f;

    u32x4 xf[D / 16];
    // the rows of x that are the wave's own, and its score tile P^T = Y X^T, masked, of the chunk in buffer buf
    auto scores = [&](int buf) {
#pragma unroll
        for (int s = 0; s < D / 16; ++s) xf[s] = frag16(&sm.x[buf][32 * it * D] + at_row[s]);
        if (tile < 0) return;
        const uint16_t* y_row = &sm.y[buf][tile == 1 ? 32 * D : 0];
        f32x16 acc;
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[r] = 0.0f;
#pragma unroll
        for (int s = 0; s < D / 16; ++s) acc = E::mfma32(frag16(y_row + at_row[s]), xf[s], acc);
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[r] *= wgt[r];
        if constexpr (kNarrow<E>) {
            const float up = power_of_scores(most_of_token(acc));
            scales.back[buf][tile][ln] = inverse_of(up);
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[r] *= up;
        }
        sm.pfrag[buf][tile][0][l] = pack_half<E>(acc, 0);
        sm.pfrag[buf][tile][1][l] = pack_half<E>(acc, 1);
    };
    scores(0);
    scale(0, 0);

    auto chunk = [&](int t, int buf) {
        const int tok0 = t * kChunk;
        const int Lc = min(kChunk, p.N - tok0);
        const int shift = kChunk - Lc;  // a ragged last chunk is right-aligned in the tile, rows above are zero

        __syncthreads();  // this chunk's scores and state are there, the last chunk's tiles are done with
        put(ahead, buf ^ 1);
        fetch(t + 2);

        // zf[f] holds tokens 16f + {4g..4g+3, 8+4g..8+4g+3} of column c_own; rows of the wave's own half in mine
        // The second term goes to the place of this chunk's rows of x, which are in registers.
        u32x4 mine[2], other[2];
        u32x4* rest = reinterpret_cast<u32x4*>(sm.x[buf]);
        auto z_frag = [&](int f) { return join(lds_tr(&sm.z[buf][16 * f * D] + z_tr[0]), lds_tr(&sm.z[buf][16 * f * D] + z_tr[1])); };
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int f = 2 * it + i;
            mine[i] = z_frag(f);
            if constexpr (kTerms < 3) {
                u32x4 zs[kTerms] = {mine[i]};
                if (kDecay) scaled<E, kTerms>(mine[i], gam_of(buf, f, 0), gam_of(buf, f, 8), zs);
                else if constexpr (kNarrow<E>) zs[0] = times_power(mine[i], scales.held[buf]);
                sm.zfrag[c][f][l] = zs[0];
                if (kTerms > 1) rest[(c * 4 + f) * 64 + l] = zs[kTerms - 1];
            }
        }
        if (it == 1)
#pragma unroll
            for (int i = 0; i < 2; ++i) other[i] = z_frag(i);

        // O^T = S^T X^T, rows of O scaled by Lam
        f32x16 o;
#pragma unroll
        for (int r = 0; r < 16; ++r) o[r] = 0.0f;
        auto lam_own = [&]() { return !kDecay ? 1.0f : shift ? sm.pw[max(32 * it + ln + later - shift, 0)] : lam_full; };
        if constexpr (kNarrow<E>) {  // the halves of the state's rows are scaled apart
            f32x16 o1 = o;
#pragma unroll
            for (int s = 0; s < D / 32; ++s) {
                o = E::mfma32(frag16(&sm.st[32 * c * D] + at_row[s]), xf[s], o);
                o1 = E::mfma32(frag16(&sm.st[32 * c * D] + at_row[D / 32 + s]), xf[D / 32 + s], o1);
            }
            const float lam = lam_own(), lam0 = scales.st_back[buf][0][c] * lam, lam1 = scales.st_back[buf][1][c] * lam;
#pragma unroll
            for (int r = 0; r < 16; ++r) o[r] = fmaf(o1[r], lam1, o[r] * lam0);
        } else {
#pragma unroll
            for (int s = 0; s < D / 16; ++s) o = E::mfma32(frag16(&sm.st[32 * c * D] + at_row[s]), xf[s], o);
            if (kDecay) {
                const float lam = lam_own();
#pragma unroll
                for (int r = 0; r < 16; ++r) o[r] *= lam;
            }
        }
        __syncthreads();  // scaled rows and the next tiles are there, everyone has read the state
        scale(buf ^ 1, buf);

        // S = gamma^L S + Y^T (Gam Z)
        if (kDecay || kNarrow<E>) {
            float gl = kDecay ? sm.pw[Lc] : 1.0f;
            if constexpr (kNarrow<E>) {
                const float next = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(scales.held[buf])));
                gl *= next * inverse_of(held);
                held = next;
            }
            if (kDecay || gl != 1.0f) {  // the same in all lanes
#pragma unroll
                for (int i = 0; i < HT; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) S[i][r] *= gl;
            }
        }
#pragma unroll
        for (int f = 0; f < 4; ++f) {
            u32x4 b[kTerms];
            if constexpr (kTerms < 3) {
                b[0] = sm.zfrag[c][f][l];
                if (kTerms > 1) b[kTerms - 1] = rest[(c * 4 + f) * 64 + l];
            } else {  // LDS has no room for the third: each wave forms all four anew
                scaled<E, kTerms>(z_frag(f), gam_of(buf, f, 0), gam_of(buf, f, 8), b);
            }
#pragma unroll
            for (int i = 0; i < HT; ++i) {
                const uint16_t* y_at = &sm.y[buf][16 * f * D];
                const u32x4 a = join(lds_tr(y_at + y_tr[i][0]), lds_tr(y_at + y_tr[i][1]));
#pragma unroll
                for (int u = 0; u < kTerms; ++u) S[i] = E::mfma32(a, b[u], S[i]);
            }
        }
        publish(buf ^ 1);

        // O^T += Z^T P^T
        auto add_tile = [&](const u32x4 (&z)[2], int n) {
            if constexpr (kNarrow<E>) {
                f32x16 acc;
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[r] = 0.0f;
#pragma unroll
                for (int hh = 0; hh < 2; ++hh) acc = E::mfma32(z[hh], sm.pfrag[buf][n][hh][l], acc);
                const float down = scales.back[buf][n][ln];
#pragma unroll
                for (int r = 0; r < 16; ++r) o[r] = fmaf(acc[r], down, o[r]);
            } else {
#pragma unroll
                for (int hh = 0; hh < 2; ++hh) o = E::mfma32(z[hh], sm.pfrag[buf][n][hh][l], o);
            }
        };
        add_tile(mine, it);
        if (it == 1) add_tile(other, 2);

        // O^T: lane = token 32it + ln, registers 4q..4q+3 = columns 32c + 8q + 4g + (0..3).  Lanes of the two halves swap
        // words, and a lane has eight neighbouring columns of its row.
        const auto to = chunk_rows(ob, D, rev, p.N, tok0);
        const int off = row_at(32 * it + ln, D, rev, shift) + (32 * c + 8 * g) * 2;
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            u32x4 val;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const u32x2 both = __builtin_amdgcn_permlane32_swap(E::pack2(o[8 * m + 2 * e], o[8 * m + 2 * e + 1]),
                                                                    E::pack2(o[8 * m + 4 + 2 * e], o[8 * m + 5 + 2 * e]), false, false);
                val[e] = both[0];
                val[2 + e] = both[1];
            }
            __builtin_amdgcn_raw_buffer_store_b128(val, to, off + 32 * m, 0, 0);  // the cache joins the pieces of a row
        }
        scores(buf ^ 1);
    };
    // two at a time without a branch between them: the loads under way are counted at every wait
    int t = 0;
    for (; t + 1 < nchunks; t += 2) {
        chunk(t, 0);
        chunk(t + 1, 1);
    }
    if (t < nchunks) chunk(t, 0);

    if (role.leave) {
        float* dst = role.leave + (size_t)unit * D * D;
        const float real = kNarrow<E> ? inverse_of(held) : 1.0f;
#pragma unroll
        for (int i = 0; i < HT; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) dst[dk_of(i, r) * D + c_own] = kNarrow<E> ? S[i][r] * real : S[i][r];
    }
}

template <typename E>
static hipError_t launch_tiles(const BwdParams& p, bool fine, hipStream_t stream) {
    const dim3 grid((p.BH + 7) / 8 * 8 * p.roles), block(SmemTiles::D * 4);
    if (!p.gamma) hipLaunchKernelGGL((tiles16_kernel<E, false, 1>), grid, block, 0, stream, p);
    else if (fine) hipLaunchKernelGGL((tiles16_kernel<E, true, 3>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((tiles16_kernel<E, true, 2>), grid, block, 0, stream, p);
    return hipGetLastError();
}

template <int D, int DV, bool kOut, typename E, bool kDecay>
static void launch_terms(const BwdParams& p, bool fine, hipStream_t stream) {
    const int units = p.BH * (kOut ? p.nseg : p.nseg - 1);
    const dim3 grid((units + 7) / 8 * 8 * p.roles), block(DV * 2);
    if constexpr (kOut) {
        if (p.N <= 2 * kChunk) {
            if constexpr (!kDecay) hipLaunchKernelGGL((walk16_kernel<D, DV, true, E, false, 1, true>), grid, block, 0, stream, p);
            else if (fine) hipLaunchKernelGGL((walk16_kernel<D, DV, true, E, true, 3, true>), grid, block, 0, stream, p);
            else hipLaunchKernelGGL((walk16_kernel<D, DV, true, E, true, 2, true>), grid, block, 0, stream, p);
            return;
        }
    }
    if constexpr (!kDecay) hipLaunchKernelGGL((walk16_kernel<D, DV, kOut, E, false, 1, false>), grid, block, 0, stream, p);
    else if (fine) hipLaunchKernelGGL((walk16_kernel<D, DV, kOut, E, true, 3, false>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((walk16_kernel<D, DV, kOut, E, true, 2, false>), grid, block, 0, stream, p);
}

template <int D, int DV, bool kOut>
static void launch_elem(const BwdParams& p, bool f16, bool fine, hipStream_t stream) {
    if (f16 && p.gamma) launch_terms<D, DV, kOut, ElemF16, true>(p, fine, stream);
    else if (f16) launch_terms<D, DV, kOut, ElemF16, false>(p, fine, stream);
    else if (p.gamma) launch_terms<D, DV, kOut, ElemBf16, true>(p, fine, stream);
    else launch_terms<D, DV, kOut, ElemBf16, false>(p, fine, stream);
}

// (D, DV) is one of (64, 64), (128, 128), (256, 128), (128, 256); the host has checked it
template <bool kOut>
static hipError_t launch_width(const BwdParams& p, int D, int DV, bool f16, bool fine, hipStream_t stream) {
    if (D == 64) launch_elem<64, 64, kOut>(p, f16, fine, stream);
    else if (D == 256) launch_elem<256, 128, kOut>(p, f16, fine, stream);
    else if (DV == 128) launch_elem<128, 128, kOut>(p, f16, fine, stream);
    else if (kOut) launch_elem<128, 256, true>(p, f16, fine, stream);
    return hipGetLastError();
}

}  // namespace bwd

hipError_t launch_bwd_16bit_states(const BwdParams& p, int D, int DV, bool f16, bool fine, hipStream_t stream) {
    return bwd::launch_width<false>(p, D, DV, f16, fine, stream);
}

hipError_t launch_bwd_16bit_walk(const BwdParams& p, int D, int DV, bool f16, bool fine, hipStream_t stream) {
    return bwd::launch_width<true>(p, D, DV, f16, fine, stream);
}

hipError_t launch_bwd_16bit_tiles(const BwdParams& p, bool f16, bool fine, hipStream_t stream) {
    return f16 ? bwd::launch_tiles<ElemF16>(p, fine, stream) : bwd::launch_tiles<ElemBf16>(p, fine, stream);
}

}  // namespace leet
