// Position rotation of query and key heads, the norm of each head with the rotation in the same pass, and that
// pass's gradient.
//
//     theta_i = position freq_i;   pair (x1, x2) -> scale (x1 cos - x2 sin, x2 cos + x1 sin)
//     y = R (w .* x r),  r = 1 / sqrt(mean(x^2) + eps)
//     du = R^T dy,  n = x r:   dx = r (w .* du - n mean(w .* du .* n)),   dw = sum of du .* n over tokens and heads
//
// Bound by memory: a row is read once and written once (2 d elements; backward 3 d).  B4 N4096 H16+16 d128 bf16: forward 51
// us, 5.3 TB/s, backward 78 us, 5.2 TB/s, where a copy of that size runs at 5.1.  Everything a row needs is arranged so
// that nothing else is read twice and no value crosses a workgroup:
//
// * A row of d elements lies in L = d / 8 neighbouring lanes, eight elements a lane in two pieces of four.  With the half
//   layout the pieces are rot / 2 apart, so both elements of every pair are in one lane; with the interleaved layout a
//   pair is within a piece.  The sums over a row are then DPP adds over L lanes.
// * A wave holds 64 / L tokens and walks over some heads of them, the next head's rows under way, so the cosines and sines,
//   which depend on the token only, are formed once a wave, in fp64.
// * Rows whose halves cannot be cut into pieces of four take the same kernel with pieces of one element (kV = 1), two pieces
//   a lane and round (rot 34 of d 128: 73, 90 and 143 us where rot 128 takes 49, 51 and 78).
#include "leet_heads.hpp"
#include "leet_io.hpp"
#include "leet_reduce.hpp"

namespace leet {

// Pieces of four elements: eight bytes of a 16-bit type.  us with pieces of four and of eight (registers: backward 94 and
// 128 with spills, forward 48 and 75): backward B4 N4096 H16+16 d128 bf16 81 and 107, forward 57 and 64.
constexpr int kPiece = 4, kPieceLog = 3;  // a row of 64 elements has 2^kPieceLog lanes
constexpr int kHeadsWaves = 4;  // waves of a workgroup
constexpr int kBackwardResident = 5;  // workgroups of the backward kernel on a compute unit
constexpr int kComputeUnits = 256;

// What a lane holds of a row: kK chunks of two pieces of kV elements, chunk k = elements first(k) .. + kV-1 and second(k)
// .. + kV-1.  The lanes' first pieces lie beside one another, and so do their second ones: an access of a wave is whole
// lines, not every other 16 bytes of them.
template <int kV, int kK, int kLog, bool kInter>
struct RowLane {
    int first[kK], second[kK];
    bool valid[kK];
    // Pairs that are rotated: of the half layout's kV pairs (a[j], b[j]) all or none; of the interleaved one's kV / 2 pairs
    // in each piece so many (one pair (a, b) where a piece is one element).
    int turned[kK], turned_b[kK];

    __device__ __forceinline__ RowLane(int lane, int d, int rot) {
#pragma unroll
        for (int k = 0; k < kK; ++k) {
            int c = (lane & ((1 << kLog) - 1)) + (k << kLog);
            valid[k] = c * 2 * kV < d;
            c = valid[k] ? c : 0;  // loads what is there, and drops it
            if (kInter && kV > 1) {
                first[k] = kV * c;
                second[k] = d / 2 + kV * c;
                turned[k] = min(max((rot - first[k]) / 2, 0), kV / 2);
                turned_b[k] = min(max((rot - second[k]) / 2, 0), kV / 2);
            } else if (kInter) {
                first[k] = 2 * c;
                second[k] = 2 * c + 1;
                turned[k] = turned_b[k] = 2 * c < rot;
            } else {
                const bool in = c * 2 * kV < rot;
                const int base = in ? 0 : rot, half = (in ? rot : d - rot) / 2;
                first[k] = base + kV * (in ? c : c - rot / (2 * kV));
                second[k] = first[k] + half;
                turned[k] = turned_b[k] = in ? kV : 0;
            }
        }
    }
};

// Sine and cosine of x in [-pi/4, pi/4] by their power series; what is left out is under 2^-36 of the sine and 2^-32.
__device__ __forceinline__ void sine_cosine(double x, double* s, double* c) {
    const double y = x * x;
    *s = fma(x * y, fma(y, fma(y, fma(y, fma(y, -1.0 / 39916800, 1.0 / 362880), -1.0 / 5040), 1.0 / 120), -1.0 / 6), x);
    *c = fma(y, fma(y, fma(y, fma(y, fma(y, -1.0 / 3628800, 1.0 / 40320), -1.0 / 720), 1.0 / 24), -0.5), 1.0);
}

// Cosines and sines (times the scale) of a lane's pairs at a position, in fp64 and rounded once.  The angle in quarter turns
// is off by some 2^-52 of itself (two products): as much as the series leave out at 2^20 radians, half a step of fp32 at 2^27.
// us with series in fp32 (up to a step off) | in fp64: B4 N4096 H16+16 d128 bf16 rotation, norm, backward 48.8 50.8 76.6 |
// 49.1 50.9 77.3, B3 N1777 H32+8 d64 fp16 11.5 13.0 23.7 | 11.4 13.6 24.1, B2 N4096 H16+4 d256 31.2 35.0 52.5 | 31.7 34.9 55.1.
template <int kV, int kK, int kLog, bool kInter>
__device__ __forceinline__ void angles(const RowLane<kV, kK, kLog, kInter>& row, const HeadsParams& p, double position,
                                       float (*cs)[kV], float (*sn)[kV]) {
    const double quarter_position = position * (2.0 / 3.14159265358979323846);
    const int turned_back = p.transposed ? 2 : 0;
#pragma unroll
    for (int k = 0; k < kK; ++k)
#pragma unroll
        for (int j = 0; j < kV; ++j) {
            const bool in_b = kInter && kV > 1 && j >= kV / 2;
            const bool in = in_b ? j - kV / 2 < row.turned_b[k] : j < row.turned[k];
            const int pair = !kInter ? row.first[k] + j : in_b ? row.second[k] / 2 + j - kV / 2 : row.first[k] / 2 + j;
            const double quarters = quarter_position * p.freq[in ? pair : 0];
            const double whole = rint(quarters);
            double s64, c64;
            sine_cosine((quarters - whole) * (3.14159265358979323846 / 2), &s64, &c64);
            const float s = (float)(s64 * (double)p.scale), c = (float)(c64 * (double)p.scale);
            // of the four quadrants only the last two bits count; a product beyond 2^31 keeps them
            const int quadrant = (int)(long long)whole;
            const float c1 = (quadrant & 1) ? s : c, s1 = (quadrant & 1) ? c : s;
            cs[k][j] = (quadrant + 1) & 2 ? -c1 : c1;
            sn[k][j] = (quadrant & 2) != turned_back ? -s1 : s1;
        }
}

// Rotates the pairs of one chunk in place.  With the half layout a pair is (a[j], b[j]), with the interleaved one two
// neighbours of a, then of b.  Elements that are not rotated keep their value, whatever their neighbour holds.
template <int kV, bool kInter>
__device__ __forceinline__ void rotate(float* a, float* b, const float* cs, const float* sn, int turned, int turned_b,
                                       float sign) {
#pragma unroll
    for (int j = 0; j < kV; ++j) {
        float* x1 = kInter ? (2 * j < kV ? a + 2 * j : b + 2 * j - kV) : a + j;
        float* x2 = kInter ? (2 * j + 1 < kV ? a + 2 * j + 1 : b + 2 * j + 1 - kV) : b + j;
        const float s = sign * sn[j];
        const float y1 = *x1 * cs[j] - *x2 * s, y2 = *x2 * cs[j] + *x1 * s;
        const bool in = kInter && kV > 1 && j >= kV / 2 ? j - kV / 2 < turned_b : j < turned;
        *x1 = in ? y1 : *x1;
        *x2 = in ? y2 : *x2;
    }
}

// A lane's part of a row as it lies in memory (at any address that suits an element: the hardware takes words anywhere).
// Loaded one head ahead, looked at when its turn comes.  kStream: with the nontemporal hint.
template <int kElem, int kV, int kK, bool kStream>
struct RawRow {
    static constexpr int kBytes = kV * Io<kElem>::kBytes;  // of a piece
    using Word = typename std::conditional<kBytes == 16, u32x4, typename std::conditional<kBytes == 8, u32x2,
                 typename std::conditional<kBytes == 4, uint32_t, uint16_t>::type>::type>::type;
    typedef Word Anywhere __attribute__((aligned(Io<kElem>::kBytes), may_alias));
    static_assert(sizeof(Word) == kBytes, "a piece is a word");
    Word a[kK], b[kK];

    static __device__ __forceinline__ Word fetch(const char* p) {
        const Anywhere* q = reinterpret_cast<const Anywhere*>(p);
        return kStream ? __builtin_nontemporal_load(q) : *q;
    }
    static __device__ __forceinline__ void put(char* p, Word w) {
        Anywhere* q = reinterpret_cast<Anywhere*>(p);
        if (kStream) __builtin_nontemporal_store(w, q);
        else *q = w;
    }
    __device__ __forceinline__ void load(const char* base, const int* first, const int* second) {
#pragma unroll
        for (int k = 0; k < kK; ++k) {
            a[k] = fetch(base + first[k] * Io<kElem>::kBytes);
            b[k] = fetch(base + second[k] * Io<kElem>::kBytes);
        }
    }
    static __device__ __forceinline__ void widen(Word w, float* f) {
        if constexpr (kElem == 0 && kV == 1) f[0] = __builtin_bit_cast(float, w);
        else if constexpr (kV == 1) f[0] = Io<kElem>::lo(w);
        else if constexpr (kElem == 0)
#pragma unroll
            for (int j = 0; j < kV; ++j) f[j] = __builtin_bit_cast(float, (uint32_t)w[j]);
        else
#pragma unroll
            for (int j = 0; j < kV / 2; ++j) {
                f[2 * j] = Io<kElem>::lo(w[j]);
                f[2 * j + 1] = Io<kElem>::hi(w[j]);
            }
    }
    static __device__ __forceinline__ Word narrow(const float* f) {
        if constexpr (kElem == 0 && kV == 1) return __builtin_bit_cast(uint32_t, f[0]);
        else if constexpr (kV == 1) return (uint16_t)Io<kElem>::pack2(f[0], 0.0f);
        else if constexpr (kElem == 0) return __builtin_bit_cast(u32x4, f32x4{f[0], f[1], f[2], f[3]});
        else return u32x2{Io<kElem>::pack2(f[0], f[1]), Io<kElem>::pack2(f[2], f[3])};
    }
    // zeros where the lane has no part of the row, or there is no row
    __device__ __forceinline__ void get(const bool* valid, bool live, float (*fa)[kV], float (*fb)[kV]) const {
#pragma unroll
        for (int k = 0; k < kK; ++k) {
            widen(a[k], fa[k]);
            widen(b[k], fb[k]);
            const bool there = live && valid[k];
#pragma unroll
            for (int j = 0; j < kV; ++j) {
                fa[k][j] = there ? fa[k][j] : 0.0f;
                fb[k][j] = there ? fb[k][j] : 0.0f;
            }
        }
    }
    static __device__ __forceinline__ void store(char* base, const int* first, const int* second, const bool* valid, bool live,
                                                 const float (*fa)[kV], const float (*fb)[kV]) {
#pragma unroll
        for (int k = 0; k < kK; ++k)
            if (live && valid[k]) {
                put(base + first[k] * Io<kElem>::kBytes, narrow(fa[k]));
                put(base + second[k] * Io<kElem>::kBytes, narrow(fb[k]));
            }
    }
};

// A lane's elements of a weight; ones where there is none.
template <int kElem, int kV, int kK>
__device__ __forceinline__ void load_weight(const void* w, bool f32, const int* first, const int* second,
                                            const bool* valid, float (*a)[kV], float (*b)[kV]) {
#pragma unroll
    for (int k = 0; k < kK; ++k)
#pragma unroll
        for (int j = 0; j < kV; ++j) {
            a[k][j] = b[k][j] = 1.0f;
            if (w && valid[k]) {
                const char* c = static_cast<const char*>(w);
                if (f32) {
                    a[k][j] = reinterpret_cast<const float*>(c)[first[k] + j];
                    b[k][j] = reinterpret_cast<const float*>(c)[second[k] + j];
                } else {
                    Io<kElem>::template load<1>(c + (first[k] + j) * Io<kElem>::kBytes, &a[k][j]);
                    Io<kElem>::template load<1>(c + (second[k] + j) * Io<kElem>::kBytes, &b[k][j]);
                }
            }
        }
}

// A row whose squares would leave fp32's range (elements beyond 2^56; or, where eps does not outweigh them, rows of a length
// below 2^-50) is multiplied by a power of two first: 1 for the others.
__device__ __forceinline__ float row_scale(float squares, float eps) {
    return squares > 0x1p120f ? 0x1p-70f : squares < 0x1p-100f && eps < 0x1p-76f ? 0x1p100f : 1.0f;
}
// Whether a wave holds such a row, or one that is not a number: a difference and a comparison of bits.  Never of fp16, whose
// sums are from 2^-48 to 2^40.  Costs nothing where rows are cut into pieces of four, 1.4 of 88 us forward and 6 of 143 backward
// in pieces of one (B4 N4096 H16+16 d128 rot 34 bf16).
template <int kElem>
__device__ __forceinline__ bool any_to_scale(float squares, float eps) {
    if (kElem == 2) return false;
    const uint32_t least = eps < 0x1p-76f ? __builtin_bit_cast(uint32_t, 0x1p-100f) : 0;
    return __any(__builtin_bit_cast(uint32_t, squares) - least > __builtin_bit_cast(uint32_t, 0x1p120f) - least);
}
template <int kK, int kV>
__device__ __forceinline__ float squares_of(const float (*a)[kV], const float (*b)[kV]) {
    float sum = 0.0f;
#pragma unroll
    for (int k = 0; k < kK; ++k)
#pragma unroll
        for (int j = 0; j < kV; ++j) sum = fmaf(a[k][j], a[k][j], fmaf(b[k][j], b[k][j], sum));
    return sum;
}
template <int kK, int kV>
__device__ __forceinline__ void times(float (*a)[kV], float (*b)[kV], float t) {
#pragma unroll
    for (int k = 0; k < kK; ++k)
#pragma unroll
        for (int j = 0; j < kV; ++j) {
            a[k][j] *= t;
            b[k][j] *= t;
        }
}

__device__ __forceinline__ double position_of(const HeadsParams& p, int b, int n) {
    return (double)(p.pos0 + (p.positions ? p.positions[b * p.positions_batch + n] : (long long)n));
}

// Forward.  Workgroup = 4 waves; wave w takes 64 / L tokens and heads_per_wave heads of the queries or of the keys.
template <int kElem, int kV, int kK, int kLog, bool kNorm, bool kInter, bool kStream>
__global__ __launch_bounds__(64 * kHeadsWaves) void heads_kernel(HeadsParams p) {
    constexpr int kTokens = 64 >> kLog;
    const int lane = threadIdx.x & 63;
    const unsigned wave = __builtin_amdgcn_readfirstlane(blockIdx.x * kHeadsWaves + (threadIdx.x >> 6));
    const unsigned unit = wave % (unsigned)p.units;
    const long long token0 = (long long)(wave / (unsigned)p.units) * kTokens;
    if (token0 >= p.tokens) return;
    const bool keys = (int)unit >= p.units_q;
    const HeadRows t = keys ? p.k : p.q;
    const int h0 = ((int)unit - (keys ? p.units_q : 0)) * p.heads_per_wave, h1 = min(h0 + p.heads_per_wave, t.H);

    const bool live = token0 + (lane >> kLog) < p.tokens;
    const int token = live ? (int)token0 + (lane >> kLog) : p.tokens - 1;
    const int b = token / p.N, n = token - b * p.N;
    const RowLane<kV, kK, kLog, kInter> row(lane, p.d, p.rot);
    const char* in = t.in + (b * t.in_b + n * t.in_n) * Io<kElem>::kBytes;
    char* out = t.out + (b * t.out_b + n * t.out_n) * Io<kElem>::kBytes;

    float wa[kK][kV], wb[kK][kV];
    if (kNorm) load_weight<kElem, kV, kK>(t.weight, p.weight_f32, row.first, row.second, row.valid, wa, wb);
    using Raw = RawRow<kElem, kV, kK, kStream>;
    Raw ahead;
    ahead.load(in + h0 * t.in_h * Io<kElem>::kBytes, row.first, row.second);
    float cs[kK][kV], sn[kK][kV];
    angles(row, p, position_of(p, b, n), cs, sn);
    for (int h = h0; h < h1; ++h) {
        float xa[kK][kV], xb[kK][kV];
        ahead.get(row.valid, live, xa, xb);
        if (h + 1 < h1) ahead.load(in + (h + 1) * t.in_h * Io<kElem>::kBytes, row.first, row.second);
        if (kNorm) {
            float sum = row_sum<kLog>(squares_of<kK, kV>(xa, xb)), eps = p.eps;
            if (__builtin_expect(any_to_scale<kElem>(sum, eps), 0)) {
                const float by = row_scale(sum, eps);
                times<kK, kV>(xa, xb, by);
                sum = row_sum<kLog>(squares_of<kK, kV>(xa, xb));
                eps = eps * by * by;
            }
            const float r = 1.0f / sqrtf(sum / (float)p.d + eps);
#pragma unroll
            for (int k = 0; k < kK; ++k)
#pragma unroll
                for (int j = 0; j < kV; ++j) {
                    xa[k][j] *= r * wa[k][j];
                    xb[k][j] *= r * wb[k][j];
                }
        }
#pragma unroll
        for (int k = 0; k < kK; ++k) rotate<kV, kInter>(xa[k], xb[k], cs[k], sn[k], row.turned[k], row.turned_b[k], 1.0f);
        Raw::store(out + h * t.out_h * Io<kElem>::kBytes, row.first, row.second, row.valid, live, xa, xb);
    }
}

// Backward.  All waves of a workgroup take the same heads (a unit); workgroup g of a unit takes token groups g, g +
// groups, ...  The lanes' sums for the weight gradient are joined over the wave's rows, then over the waves, and go to
// one row of `partial`; heads_weight_kernel adds the rows up in order.
// plan_heads launches five workgroups a compute unit, which leaves 96 registers a lane.  Rows of 16 bits fit (but for two or
// three words a lane at width 256, which the kernel leaves in scratch memory), rows of fp32 leave nine to thirteen words
// there: four workgroups would take 108 registers and nothing there, in as much time (us with five | four: B2 N2047 H8+8 d64 fp32
// 17.3 16.8, B2 N4096 H16+16 d128 fp32 77.8 75.6, the same in bf16 with N4096 B4 79.7 81.0, d256 H16+4 56.3 58.9).
template <int kElem, int kV, int kK, int kLog, bool kInter, bool kStream>
__global__ __launch_bounds__(64 * kHeadsWaves, kBackwardResident) void heads_backward_kernel(HeadsParams p) {
    constexpr int kTokens = 64 >> kLog;
    __shared__ float joined[kHeadsWaves][kK][2 * kV][1 << kLog];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int unit = (int)(blockIdx.x % (unsigned)p.units), group = (int)(blockIdx.x / (unsigned)p.units);
    const bool keys = unit >= p.units_q;
    const HeadRows t = keys ? p.k : p.q;
    const int h0 = (unit - (keys ? p.units_q : 0)) * p.heads_per_wave, h1 = min(h0 + p.heads_per_wave, t.H);
    using Raw = RawRow<kElem, kV, kK, kStream>;
    const RowLane<kV, kK, kLog, kInter> row(lane, p.d, p.rot);
    float wa[kK][kV], wb[kK][kV], ga[kK][kV], gb[kK][kV];
    load_weight<kElem, kV, kK>(t.weight, p.weight_f32, row.first, row.second, row.valid, wa, wb);
#pragma unroll
    for (int k = 0; k < kK; ++k)
#pragma unroll
        for (int j = 0; j < kV; ++j) ga[k][j] = gb[k][j] = 0.0f;

    const long long step = (long long)p.groups * kHeadsWaves * kTokens;
    for (long long token0 = ((long long)group * kHeadsWaves + wave) * kTokens; token0 < p.tokens; token0 += step) {
        const bool live = token0 + (lane >> kLog) < p.tokens;
        const int token = live ? (int)token0 + (lane >> kLog) : p.tokens - 1;
        const int b = token / p.N, n = token - b * p.N;
        const char* in = t.in + (b * t.in_b + n * t.in_n) * Io<kElem>::kBytes;
        const char* grad = t.grad + (b * t.grad_b + n * t.grad_n) * Io<kElem>::kBytes;
        char* out = t.out + (b * t.out_b + n * t.out_n) * Io<kElem>::kBytes;
        Raw ahead_x, ahead_u;
        ahead_x.load(in + h0 * t.in_h * Io<kElem>::kBytes, row.first, row.second);
        ahead_u.load(grad + h0 * t.grad_h * Io<kElem>::kBytes, row.first, row.second);
        float cs[kK][kV], sn[kK][kV];
        angles(row, p, position_of(p, b, n), cs, sn);
        for (int h = h0; h < h1; ++h) {
            float xa[kK][kV], xb[kK][kV], ua[kK][kV], ub[kK][kV];
            ahead_x.get(row.valid, live, xa, xb);
            ahead_u.get(row.valid, live, ua, ub);
            if (h + 1 < h1) {
                ahead_x.load(in + (h + 1) * t.in_h * Io<kElem>::kBytes, row.first, row.second);
                ahead_u.load(grad + (h + 1) * t.grad_h * Io<kElem>::kBytes, row.first, row.second);
            }
#pragma unroll
            for (int k = 0; k < kK; ++k)
                rotate<kV, kInter>(ua[k], ub[k], cs[k], sn[k], row.turned[k], row.turned_b[k], -1.0f);
            auto dot_of = [&] {
                float dot = 0.0f;
#pragma unroll
                for (int k = 0; k < kK; ++k)
#pragma unroll
                    for (int j = 0; j < kV; ++j)
                        dot = fmaf(ua[k][j] * wa[k][j], xa[k][j], fmaf(ub[k][j] * wb[k][j], xb[k][j], dot));
                return row_sum<kLog>(dot);
            };
            float sum = row_sum<kLog>(squares_of<kK, kV>(xa, xb)), dot = dot_of(), eps = p.eps, by = 1.0f;
            const bool scaled = any_to_scale<kElem>(sum, eps);
            if (__builtin_expect(scaled, 0)) {
                by = row_scale(sum, eps);
                times<kK, kV>(xa, xb, by);
                sum = row_sum<kLog>(squares_of<kK, kV>(xa, xb));
                dot = dot_of();
                eps = eps * by * by;
            }
            const float r = 1.0f / sqrtf(sum / (float)p.d + eps);
            const float mean = r * dot / (float)p.d;  // of w du n
#pragma unroll
            for (int k = 0; k < kK; ++k)
#pragma unroll
                for (int j = 0; j < kV; ++j) {
                    const float na = xa[k][j] * r, nb = xb[k][j] * r;
                    // rows past the last token hold zeros, and 0 times an infinite r must not count
                    ga[k][j] += live ? ua[k][j] * na : 0.0f;
                    gb[k][j] += live ? ub[k][j] * nb : 0.0f;
                    xa[k][j] = r * (ua[k][j] * wa[k][j] - na * mean);
                    xb[k][j] = r * (ub[k][j] * wb[k][j] - nb * mean);
                }
            if (__builtin_expect(scaled, 0)) times<kK, kV>(xa, xb, by);  // r is that of the scaled row
            Raw::store(out + h * t.out_h * Io<kElem>::kBytes, row.first, row.second, row.valid, live, xa, xb);
        }
    }
    if (!p.partial) return;
#pragma unroll
    for (int k = 0; k < kK; ++k)
#pragma unroll
        for (int j = 0; j < kV; ++j) {
#pragma unroll
            for (int off = 1 << kLog; off < 64; off <<= 1) {
                ga[k][j] += __shfl_xor(ga[k][j], off, 64);
                gb[k][j] += __shfl_xor(gb[k][j], off, 64);
            }
            if (lane < (1 << kLog)) {
                joined[wave][k][j][lane] = ga[k][j];
                joined[wave][k][kV + j][lane] = gb[k][j];
            }
        }
    __syncthreads();
    if (wave == 0 && lane < (1 << kLog)) {
        // rows of `partial`: the queries' workgroups, then the keys'
        const int units_k = p.units - p.units_q;
        float* to = p.partial + (size_t)(keys ? p.groups * p.units_q + group * units_k + unit - p.units_q
                                              : group * p.units_q + unit) * p.d;
#pragma unroll
        for (int k = 0; k < kK; ++k)
            if (row.valid[k])
#pragma unroll
                for (int j = 0; j < kV; ++j) {
                    float a = 0.0f, b = 0.0f;
#pragma unroll
                    for (int v = 0; v < kHeadsWaves; ++v) {
                        a += joined[v][k][j][lane];
                        b += joined[v][k][kV + j][lane];
                    }
                    to[row.first[k] + j] = a;
                    to[row.second[k] + j] = b;
                }
    }
}

// dw = sum of the rows of `partial`, queries (blockIdx.y = 0) and keys (1).  Workgroup = 16 columns x 64 row groups;
// each thread adds its rows in order, the groups are joined in a fixed tree.
constexpr int kSumColumns = 16, kSumGroups = 64;
template <int kElem>
__global__ __launch_bounds__(kSumColumns * kSumGroups) void heads_weight_kernel(HeadsParams p) {
    __shared__ float part[kSumGroups][kSumColumns + 1];
    const bool keys = blockIdx.y != 0;
    void* to = keys ? p.k.weight_grad : p.q.weight_grad;
    if (!to) return;
    const int c = threadIdx.x % kSumColumns, g = threadIdx.x / kSumColumns, col = blockIdx.x * kSumColumns + c;
    const int rows_q = p.groups * p.units_q, first = keys ? rows_q : 0;
    const int rows = keys ? p.groups * (p.units - p.units_q) : rows_q;
    float sum = 0.0f;
    if (col < p.d)
#pragma unroll 8
        for (int r = g; r < rows; r += kSumGroups) sum += p.partial[(size_t)(first + r) * p.d + col];
    part[g][c] = sum;
    __syncthreads();
    for (int half = kSumGroups / 2; half > 0; half /= 2) {
        if (g < half) part[g][c] += part[g + half][c];
        __syncthreads();
    }
    if (g == 0 && col < p.d) {
        const float v = part[0][c];
        if (p.weight_f32) static_cast<float*>(to)[col] = v;
        else Io<kElem>::template store<1>(static_cast<char*>(to) + (size_t)col * Io<kElem>::kBytes, &v);
    }
}

// Lanes of a row, as a power of two: d / 8 and more with pieces of four, a whole wave with pieces of one.
static int row_log(const HeadsParams& p) { return !p.vector ? 6 : kPieceLog + (p.d <= 64 ? 0 : p.d <= 128 ? 1 : 2); }

// Heads a wave takes: the more, the fewer angles are formed twice; the fewer, the more waves there are.  Rows from memory
// want 64 waves a compute unit (16 and 64: forward B4 N4096 H16+16 d128 57 and 51 us, backward 92 and 78), rows from the
// cache 16 (forward B3 N1777 H32+8 d64 with 4, 16, 64: 14.8 13.3 18, B4 N1024 H16+16 d128 15.3 13.7 -) or, backward, where a
// workgroup ends with a sum over its waves, 4 (B2 N2047 H8+8 d64 fp32 with 4, 16, 32: 14.8 18.4 20.7, B4 N1024 H16+16 d128
// 24.3 23.7 23.4).
// Elsewhere, us with 4 | 16 | 64: forward from the cache B1 N2048 H32+8 d128 bf16 14.9 11.9 20, B2 N1500 H24+24 d80 16.3 15.1
// 19.6; from memory with 16 | 64: B1 N16384 H32+8 d128 66.5 63.7, B2 N4096 H16+16 d128 fp32 48.7 51.6, B16 N2048 H12+12 d64 fp16
// 49.9 49.9.  Backward, where the rule is less good, from the cache with 4 | 16: the first two 23.9 19.9 and 28.3 24.5; from
// memory with 16 | 64: the last three 104 99, 79.1 77.9, 76.7 92.3.
void plan_heads(HeadsParams* p, bool backward) {
    const long tokens = 64 >> row_log(*p);
    const long groups = (p->tokens + tokens - 1) / tokens;  // waves that one head a wave needs
    const long want = (p->stream ? 64 : backward ? 4 : 16) * kComputeUnits;
    const int most = p->q.H > p->k.H ? p->q.H : p->k.H;
    int heads = 16;
    while (heads > 1 && groups * ((p->q.H + heads - 1) / heads + (p->k.H + heads - 1) / heads) < want) heads /= 2;
    if (heads > most) heads = most;
    p->heads_per_wave = heads;
    p->units_q = (p->q.H + heads - 1) / heads;
    p->units = p->units_q + (p->k.H + heads - 1) / heads;
    if (backward) {
        const long blocks = (groups + kHeadsWaves - 1) / kHeadsWaves;
        long most_groups = kBackwardResident * kComputeUnits / p->units;
        if (most_groups < 1) most_groups = 1;
        p->groups = (int)(blocks < most_groups ? blocks : most_groups);
    }
}

template <int kElem, int kV, int kK, int kLog, bool kNorm, bool kStream>
static void launch_heads_l(const HeadsParams& p, int layout, hipStream_t stream) {
    const long long waves = (((long long)p.tokens + (64 >> kLog) - 1) >> (6 - kLog)) * p.units;
    const dim3 grid((unsigned)((waves + kHeadsWaves - 1) / kHeadsWaves)), block(64 * kHeadsWaves);
    if (layout) hipLaunchKernelGGL((heads_kernel<kElem, kV, kK, kLog, kNorm, true, kStream>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((heads_kernel<kElem, kV, kK, kLog, kNorm, false, kStream>), grid, block, 0, stream, p);
}

template <int kElem, bool kNorm, bool kStream>
static void launch_heads_s(const HeadsParams& p, int layout, hipStream_t stream) {
    const int log = row_log(p);
    if (log == kPieceLog) launch_heads_l<kElem, kPiece, 1, kPieceLog, kNorm, kStream>(p, layout, stream);
    else if (log == kPieceLog + 1) launch_heads_l<kElem, kPiece, 1, kPieceLog + 1, kNorm, kStream>(p, layout, stream);
    else launch_heads_l<kElem, kPiece, 1, kPieceLog + 2, kNorm, kStream>(p, layout, stream);
}

template <int kElem, bool kNorm>
static hipError_t launch_heads_e(const HeadsParams& p, int layout, hipStream_t stream) {
    if (!p.vector) launch_heads_l<kElem, 1, 2, 6, kNorm, false>(p, layout, stream);
    else if (p.stream) launch_heads_s<kElem, kNorm, true>(p, layout, stream);
    else launch_heads_s<kElem, kNorm, false>(p, layout, stream);
    return hipGetLastError();
}

hipError_t launch_heads(const HeadsParams& p, int elem, int layout, bool norm, hipStream_t stream) {
    if (norm)
        return elem == 0 ? launch_heads_e<0, true>(p, layout, stream)
             : elem == 1 ? launch_heads_e<1, true>(p, layout, stream)
                         : launch_heads_e<2, true>(p, layout, stream);
    return elem == 0 ? launch_heads_e<0, false>(p, layout, stream)
         : elem == 1 ? launch_heads_e<1, false>(p, layout, stream)
                     : launch_heads_e<2, false>(p, layout, stream);
}

template <int kElem, int kV, int kK, int kLog, bool kStream>
static void launch_heads_backward_l(const HeadsParams& p, int layout, hipStream_t stream) {
    const dim3 grid((unsigned)(p.groups * p.units)), block(64 * kHeadsWaves);
    if (layout) hipLaunchKernelGGL((heads_backward_kernel<kElem, kV, kK, kLog, true, kStream>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((heads_backward_kernel<kElem, kV, kK, kLog, false, kStream>), grid, block, 0, stream, p);
}

template <int kElem, bool kStream>
static void launch_heads_backward_s(const HeadsParams& p, int layout, hipStream_t stream) {
    const int log = row_log(p);
    if (log == kPieceLog) launch_heads_backward_l<kElem, kPiece, 1, kPieceLog, kStream>(p, layout, stream);
    else if (log == kPieceLog + 1) launch_heads_backward_l<kElem, kPiece, 1, kPieceLog + 1, kStream>(p, layout, stream);
    else launch_heads_backward_l<kElem, kPiece, 1, kPieceLog + 2, kStream>(p, layout, stream);
}

template <int kElem>
static hipError_t launch_heads_backward_e(const HeadsParams& p, int layout, hipStream_t stream) {
    if (!p.vector) launch_heads_backward_l<kElem, 1, 2, 6, false>(p, layout, stream);
    else if (p.stream) launch_heads_backward_s<kElem, true>(p, layout, stream);
    else launch_heads_backward_s<kElem, false>(p, layout, stream);
    return hipGetLastError();
}

hipError_t launch_heads_backward(const HeadsParams& p, int elem, int layout, hipStream_t stream) {
    return elem == 0 ? launch_heads_backward_e<0>(p, layout, stream)
         : elem == 1 ? launch_heads_backward_e<1>(p, layout, stream)
                     : launch_heads_backward_e<2>(p, layout, stream);
}

hipError_t launch_heads_weights(const HeadsParams& p, int elem, hipStream_t stream) {
    const dim3 grid((unsigned)((p.d + kSumColumns - 1) / kSumColumns), 2), block(kSumColumns * kSumGroups);
    if (elem == 0) hipLaunchKernelGGL((heads_weight_kernel<0>), grid, block, 0, stream, p);
    else if (elem == 1) hipLaunchKernelGGL((heads_weight_kernel<1>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((heads_weight_kernel<2>), grid, block, 0, stream, p);
    return hipGetLastError();
}

}  // namespace leet
