// Position rotation of query and key heads, the norm of each head with the rotation in the same pass, and that
// pass's gradient.
//
//     theta_i = position freq_i;   pair (x1, x2) -> scale (x1 cos - x2 sin, x2 cos + x1 sin)
//     y = R (w .* x r),  r = 1 / sqrt(mean(x^2) + eps)
//     du = R^T dy,  n = x r:   dx = r (w .* du - n mean(w .* du .* n)),   dw = sum of du .* n over tokens and heads
//
// Bound by memory: a row is read once and written once (2 d elements; backward 3 d).  Everything a row needs is
// arranged so that nothing else is read twice and no value crosses a workgroup:
//
// * A row of d elements lies in L = d / 16 neighbouring lanes, sixteen elements a lane in two pieces of eight (two
//   16-byte accesses of a 16-bit type).  With the half layout the pieces are rot / 2 apart, so both elements of every
//   pair are in one lane; with the interleaved layout they are adjacent.  The sums over a row are then DPP adds over
//   L lanes.
// * A wave holds 64 / L tokens and walks over some heads of them, so the cosines and sines, which depend on the token
//   only, are formed once a wave: in fp64 up to the reduced angle (a product, two roundings), in fp32 from there.
// * Rows that are not 16-byte aligned, or whose halves cannot be cut into pieces of eight, take the same kernel with
//   pieces of one element (kV = 1), two pieces a lane and round.
#include "leet_heads.hpp"
#include "leet_io.hpp"

namespace leet {

constexpr int kHeadsWaves = 4;  // waves of a workgroup
constexpr double kInvTwoPi = 0.15915494309189533576888;

// Sum over the 2^kLog neighbouring lanes that hold a row; every one of them gets it, with the same bits.
template <int kCtrl>
__device__ __forceinline__ float dpp(float x) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), kCtrl, 0xf, 0xf, true));
}
template <int kLog>
__device__ __forceinline__ float row_sum(float v) {
    if constexpr (kLog >= 1) v += dpp<0xB1>(v);   // quad_perm 1 0 3 2
    if constexpr (kLog >= 2) v += dpp<0x4E>(v);   // quad_perm 2 3 0 1
    if constexpr (kLog >= 3) v += dpp<0x141>(v);  // row_half_mirror: the quads of eight lanes swap
    if constexpr (kLog >= 4) v += dpp<0x140>(v);  // row_mirror: the halves of sixteen lanes swap
    if constexpr (kLog >= 5) v += __shfl_xor(v, 16, 64);
    if constexpr (kLog >= 6) v += __shfl_xor(v, 32, 64);
    return v;
}

// What a lane holds of a row: kK chunks of 2 kV elements, chunk k = elements first(k) .. + kV-1 and second(k) .. + kV-1.
template <int kV, int kK, int kLog, bool kInter>
struct RowLane {
    int first[kK], second[kK];
    bool valid[kK];
    int turned[kK];  // pairs of the chunk that are rotated (with the half layout all or none)

    __device__ __forceinline__ RowLane(int lane, int d, int rot) {
#pragma unroll
        for (int k = 0; k < kK; ++k) {
            const int c = (lane & ((1 << kLog) - 1)) + (k << kLog);
            valid[k] = c * 2 * kV < d;
            if (kInter) {
                first[k] = 2 * kV * c;
                second[k] = first[k] + kV;
                turned[k] = min(max(rot / 2 - kV * c, 0), kV);
            } else {
                const bool in = c * 2 * kV < rot;
                first[k] = in ? kV * c : 2 * kV * c;
                second[k] = in ? rot / 2 + kV * c : 2 * kV * c + kV;
                turned[k] = in ? kV : 0;
            }
        }
    }
};

// Cosines and sines (times the scale) of a lane's pairs at a position.  The angle in turns is a product in fp64; its
// distance to the nearest quarter turn is at most an eighth and goes on in fp32, where it is off by 2^-28 of a turn at
// most, so a cosine is off by little more than its own rounding however far out the position is.
template <int kV, int kK, int kLog, bool kInter>
__device__ __forceinline__ void angles(const RowLane<kV, kK, kLog, kInter>& row, const HeadsParams& p, double position,
                                       float (*cs)[kV], float (*sn)[kV]) {
#pragma unroll
    for (int k = 0; k < kK; ++k)
#pragma unroll
        for (int j = 0; j < kV; ++j) {
            cs[k][j] = 1.0f;
            sn[k][j] = 0.0f;
            if (j < row.turned[k]) {
                const int pair = kInter ? row.first[k] / 2 + j : row.first[k] + j;
                const double quarters = position * (p.freq[pair] * (4.0 * kInvTwoPi));
                const double whole = rint(quarters);
                const int quadrant = (int)(long long)whole & 3;
                float s, c;
                sincospif(0.5f * (float)(quarters - whole), &s, &c);
                const float c1 = (quadrant & 1) ? s : c, s1 = (quadrant & 1) ? c : s;
                cs[k][j] = (quadrant == 1 || quadrant == 2 ? -c1 : c1) * p.scale;
                const float sv = (quadrant >= 2 ? -s1 : s1) * p.scale;
                sn[k][j] = p.transposed ? -sv : sv;
            }
        }
}

// Rotates the pairs of one chunk in place.  With the half layout a pair is (a[j], b[j]), with the interleaved one two
// neighbours of a, then of b.  Elements that are not rotated keep their value, whatever their neighbour holds.
template <int kV, bool kInter>
__device__ __forceinline__ void rotate(float* a, float* b, const float* cs, const float* sn, int turned, float sign) {
#pragma unroll
    for (int j = 0; j < kV; ++j) {
        float* x1 = kInter ? (2 * j < kV ? a + 2 * j : b + 2 * j - kV) : a + j;
        float* x2 = kInter ? (2 * j + 1 < kV ? a + 2 * j + 1 : b + 2 * j + 1 - kV) : b + j;
        const float s = sign * sn[j];
        const float y1 = *x1 * cs[j] - *x2 * s, y2 = *x2 * cs[j] + *x1 * s;
        *x1 = j < turned ? y1 : *x1;
        *x2 = j < turned ? y2 : *x2;
    }
}

template <int kElem, int kV, int kK>
__device__ __forceinline__ void load_row(const char* base, const int* first, const int* second, const bool* valid,
                                         bool live, float (*a)[kV], float (*b)[kV]) {
#pragma unroll
    for (int k = 0; k < kK; ++k) {
        if (live && valid[k]) {
            Io<kElem>::template load<kV>(base + (long long)first[k] * Io<kElem>::kBytes, a[k]);
            Io<kElem>::template load<kV>(base + (long long)second[k] * Io<kElem>::kBytes, b[k]);
        } else {
#pragma unroll
            for (int j = 0; j < kV; ++j) a[k][j] = b[k][j] = 0.0f;
        }
    }
}

template <int kElem, int kV, int kK>
__device__ __forceinline__ void store_row(char* base, const int* first, const int* second, const bool* valid, bool live,
                                          const float (*a)[kV], const float (*b)[kV]) {
#pragma unroll
    for (int k = 0; k < kK; ++k)
        if (live && valid[k]) {
            Io<kElem>::template store<kV>(base + (long long)first[k] * Io<kElem>::kBytes, a[k]);
            Io<kElem>::template store<kV>(base + (long long)second[k] * Io<kElem>::kBytes, b[k]);
        }
}

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

__device__ __forceinline__ double position_of(const HeadsParams& p, int b, int n) {
    return (double)(p.pos0 + (p.positions ? p.positions[b * p.positions_batch + n] : (long long)n));
}

// Forward.  Workgroup = 4 waves; wave w takes 64 / L tokens and heads_per_wave heads of the queries or of the keys.
template <int kElem, int kV, int kK, int kLog, bool kNorm, bool kInter>
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
    float cs[kK][kV], sn[kK][kV];
    angles(row, p, position_of(p, b, n), cs, sn);

    for (int h = h0; h < h1; ++h) {
        float xa[kK][kV], xb[kK][kV];
        load_row<kElem, kV, kK>(in + h * t.in_h * Io<kElem>::kBytes, row.first, row.second, row.valid, live, xa, xb);
        if (kNorm) {
            float sum = 0.0f;
#pragma unroll
            for (int k = 0; k < kK; ++k)
#pragma unroll
                for (int j = 0; j < kV; ++j) sum = fmaf(xa[k][j], xa[k][j], fmaf(xb[k][j], xb[k][j], sum));
            const float r = 1.0f / sqrtf(row_sum<kLog>(sum) / (float)p.d + p.eps);
#pragma unroll
            for (int k = 0; k < kK; ++k)
#pragma unroll
                for (int j = 0; j < kV; ++j) {
                    xa[k][j] *= r * wa[k][j];
                    xb[k][j] *= r * wb[k][j];
                }
        }
#pragma unroll
        for (int k = 0; k < kK; ++k) rotate<kV, kInter>(xa[k], xb[k], cs[k], sn[k], row.turned[k], 1.0f);
        store_row<kElem, kV, kK>(out + h * t.out_h * Io<kElem>::kBytes, row.first, row.second, row.valid, live, xa, xb);
    }
}

// Backward.  All waves of a workgroup take the same heads (a unit); workgroup g of a unit takes token groups g, g +
// groups, ...  The lanes' sums for the weight gradient are joined over the wave's rows, then over the waves, and go to
// one row of `partial`; heads_weight_kernel adds the rows up in order.
template <int kElem, int kV, int kK, int kLog, bool kInter>
__global__ __launch_bounds__(64 * kHeadsWaves) void heads_backward_kernel(HeadsParams p) {
    constexpr int kTokens = 64 >> kLog;
    __shared__ float joined[kHeadsWaves][kK][2 * kV][1 << kLog];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int unit = (int)(blockIdx.x % (unsigned)p.units), group = (int)(blockIdx.x / (unsigned)p.units);
    const bool keys = unit >= p.units_q;
    const HeadRows t = keys ? p.k : p.q;
    const int h0 = (unit - (keys ? p.units_q : 0)) * p.heads_per_wave, h1 = min(h0 + p.heads_per_wave, t.H);
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
        float cs[kK][kV], sn[kK][kV];
        angles(row, p, position_of(p, b, n), cs, sn);
        for (int h = h0; h < h1; ++h) {
            float xa[kK][kV], xb[kK][kV], ua[kK][kV], ub[kK][kV];
            load_row<kElem, kV, kK>(in + h * t.in_h * Io<kElem>::kBytes, row.first, row.second, row.valid, live, xa, xb);
            load_row<kElem, kV, kK>(grad + h * t.grad_h * Io<kElem>::kBytes, row.first, row.second, row.valid, live, ua, ub);
            float sum = 0.0f, dot = 0.0f;
#pragma unroll
            for (int k = 0; k < kK; ++k) {
                rotate<kV, kInter>(ua[k], ub[k], cs[k], sn[k], row.turned[k], -1.0f);
#pragma unroll
                for (int j = 0; j < kV; ++j) {
                    sum = fmaf(xa[k][j], xa[k][j], fmaf(xb[k][j], xb[k][j], sum));
                    dot = fmaf(ua[k][j] * wa[k][j], xa[k][j], fmaf(ub[k][j] * wb[k][j], xb[k][j], dot));
                }
            }
            const float r = 1.0f / sqrtf(row_sum<kLog>(sum) / (float)p.d + p.eps);
            const float mean = r * row_sum<kLog>(dot) / (float)p.d;  // of w du n
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
            store_row<kElem, kV, kK>(out + h * t.out_h * Io<kElem>::kBytes, row.first, row.second, row.valid, live, xa, xb);
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

// Lanes of a row: d / 16 with pieces of eight (d a multiple of 16: 1, 2, 4, 8 or 16 lanes, the next power of two), a
// whole wave with pieces of one.
static int row_log(const HeadsParams& p) { return !p.vector ? 6 : p.d <= 64 ? 2 : p.d <= 128 ? 3 : 4; }

void plan_heads(HeadsParams* p, bool backward) {
    const long tokens = 64 >> row_log(*p);
    const long groups = (p->tokens + tokens - 1) / tokens;  // waves that one head a wave needs
    // Heads a wave: as many as leave about 16 waves a compute unit, 16 at most; the more, the fewer angles are formed twice.
    const int most = p->q.H > p->k.H ? p->q.H : p->k.H;
    int heads = 16;
    while (heads > 1 && groups * ((p->q.H + heads - 1) / heads + (p->k.H + heads - 1) / heads) < 4096) heads /= 2;
    if (heads > most) heads = most;
    p->heads_per_wave = heads;
    p->units_q = (p->q.H + heads - 1) / heads;
    p->units = p->units_q + (p->k.H + heads - 1) / heads;
    if (backward) {
        const long blocks = (groups + kHeadsWaves - 1) / kHeadsWaves;
        long want = 1024 / p->units;
        if (want < 1) want = 1;
        p->groups = (int)(blocks < want ? blocks : want);
    }
}

template <int kElem, int kV, int kK, int kLog, bool kNorm>
static void launch_heads_l(const HeadsParams& p, int layout, unsigned blocks, hipStream_t stream) {
    const dim3 grid(blocks), block(64 * kHeadsWaves);
    if (layout) hipLaunchKernelGGL((heads_kernel<kElem, kV, kK, kLog, kNorm, true>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((heads_kernel<kElem, kV, kK, kLog, kNorm, false>), grid, block, 0, stream, p);
}

template <int kElem, bool kNorm>
static void launch_heads_e(const HeadsParams& p, int layout, hipStream_t stream) {
    const int log = row_log(p);
    const long long waves = (((long long)p.tokens + (64 >> log) - 1) >> (6 - log)) * p.units;
    const unsigned blocks = (unsigned)((waves + kHeadsWaves - 1) / kHeadsWaves);
    if (log == 2) launch_heads_l<kElem, 8, 1, 2, kNorm>(p, layout, blocks, stream);
    else if (log == 3) launch_heads_l<kElem, 8, 1, 3, kNorm>(p, layout, blocks, stream);
    else if (log == 4) launch_heads_l<kElem, 8, 1, 4, kNorm>(p, layout, blocks, stream);
    else launch_heads_l<kElem, 1, 2, 6, kNorm>(p, layout, blocks, stream);
}

hipError_t launch_heads(const HeadsParams& p, int elem, int layout, bool norm, hipStream_t stream) {
    if (norm) {
        if (elem == 0) launch_heads_e<0, true>(p, layout, stream);
        else if (elem == 1) launch_heads_e<1, true>(p, layout, stream);
        else launch_heads_e<2, true>(p, layout, stream);
    } else {
        if (elem == 0) launch_heads_e<0, false>(p, layout, stream);
        else if (elem == 1) launch_heads_e<1, false>(p, layout, stream);
        else launch_heads_e<2, false>(p, layout, stream);
    }
    return hipGetLastError();
}

template <int kElem, int kV, int kK, int kLog>
static void launch_heads_backward_l(const HeadsParams& p, int layout, hipStream_t stream) {
    const dim3 grid((unsigned)(p.groups * p.units)), block(64 * kHeadsWaves);
    if (layout) hipLaunchKernelGGL((heads_backward_kernel<kElem, kV, kK, kLog, true>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((heads_backward_kernel<kElem, kV, kK, kLog, false>), grid, block, 0, stream, p);
}

template <int kElem>
static hipError_t launch_heads_backward_e(const HeadsParams& p, int layout, hipStream_t stream) {
    const int log = row_log(p);
    if (log == 2) launch_heads_backward_l<kElem, 8, 1, 2>(p, layout, stream);
    else if (log == 3) launch_heads_backward_l<kElem, 8, 1, 3>(p, layout, stream);
    else if (log == 4) launch_heads_backward_l<kElem, 8, 1, 4>(p, layout, stream);
    else launch_heads_backward_l<kElem, 1, 2, 6>(p, layout, stream);
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
