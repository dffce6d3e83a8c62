// Norm of rows of a residual stream, with the stream's addition in the same pass and an output in 8 bits with scales, and its
// gradient.
//
//     s = x + residual,   y = w .* s r,   r = 1 / sqrt(mean(s^2) + eps);      8 bits: scale = max |y| / 448, q = e4m3(y / scale)
//     dh = r (w .* dy - n mean(w .* dy .* n)) + what comes along the stream,   n = h r,   dw = sum of dy .* n over the rows
//
// Bound by memory: every row is read once and written once.  A row of up to 8 T channels lies in T threads' registers, eight
// neighbouring channels a thread, T the least of 64 .. 1024 that holds it (twice eight beyond 8192 channels).  One wave takes a
// row of up to 512 channels by itself, else a workgroup, whose waves' sums meet in LDS at one barrier.  bf16 with a residual, 16384
// rows of 2048: 48 us, 5.6 TB/s, backward 51 and 4.5 for the weight's; 14216 rows of 4096 with an fp32 stream to 8 bits 115 us, 5.6 TB/s;
// one row of 4096 2.4 us.
#include "leet_io.hpp"
#include "leet_norm.hpp"
#include "leet_reduce.hpp"

namespace leet {

constexpr float kE4m3Most = 448.0f;
constexpr float kLeast = 0x1p-100f;  // a scale is made for no less than this: rows of zeros have one, and 1 / scale is finite

// Eight neighbouring elements as they lie in memory, at any address that suits one; the last ones of a row may be fewer.
template <int kElem, bool kFar>
struct Eight {
    static constexpr int kWords = kElem == 0 ? 2 : 1, kBytes = Io<kElem>::kBytes;
    using Word = typename std::conditional<kElem == 0, u32x4, u32x4>::type;  // a dependent type, for an alignment that is one
    typedef Word Anywhere __attribute__((aligned(kBytes), may_alias));
    u32x4 word[kWords];

    __device__ __forceinline__ void load(const char* p, int count) {
        if (count >= 8) {
#pragma unroll
            for (int i = 0; i < kWords; ++i) {
                const Anywhere* q = reinterpret_cast<const Anywhere*>(p) + i;
                word[i] = kFar ? __builtin_nontemporal_load(q) : *q;
            }
        } else {
#pragma unroll
            for (int i = 0; i < kWords; ++i) word[i] = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
            for (int j = 0; j < 7; ++j)
                if (j < count) {
                    if constexpr (kElem == 0) word[j >> 2][j & 3] = reinterpret_cast<const uint32_t*>(p)[j];
                    else word[0][j >> 1] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[j] << (16 * (j & 1));
                }
        }
    }
    __device__ __forceinline__ void get(float (&f)[8]) const {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (kElem == 0) {
                f[j] = __builtin_bit_cast(float, (uint32_t)word[0][j]);
                f[4 + j] = __builtin_bit_cast(float, (uint32_t)word[kWords - 1][j]);
            } else {
                f[2 * j] = Io<kElem>::lo(word[0][j]);
                f[2 * j + 1] = Io<kElem>::hi(word[0][j]);
            }
        }
    }
    static __device__ __forceinline__ void store(char* p, int count, const float (&f)[8]) {
        if (count >= 8) {
            if constexpr (kElem == 0) {
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    put(p + 16 * i, __builtin_bit_cast(u32x4, f32x4{f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]}));
            } else {
                put(p, u32x4{Io<kElem>::pack2(f[0], f[1]), Io<kElem>::pack2(f[2], f[3]), Io<kElem>::pack2(f[4], f[5]),
                             Io<kElem>::pack2(f[6], f[7])});
            }
        } else {
#pragma unroll
            for (int j = 0; j < 7; ++j)
                if (j < count) Io<kElem>::template store<1>(p + j * kBytes, &f[j]);
        }
    }
    static __device__ __forceinline__ void put(char* p, u32x4 w) {
        Anywhere* q = reinterpret_cast<Anywhere*>(p);
        if (kFar) __builtin_nontemporal_store(w, q);
        else *q = w;
    }
};

// Eight channels of a weight; ones where there is none.
template <int kElem>
__device__ __forceinline__ void load_weights(const NormParams& p, int first, int count, float (&w)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = 1.0f;
    if (!p.weight) return;
    if (p.weight_f32) {
        Eight<0, false> raw;
        raw.load(static_cast<const char*>(p.weight) + (size_t)first * 4, count);
        raw.get(w);
    } else {
        Eight<kElem, false> raw;
        raw.load(static_cast<const char*>(p.weight) + (size_t)first * Io<kElem>::kBytes, count);
        raw.get(w);
    }
}

// A row whose squares would leave fp32's range is multiplied by a power of two first: 1 for the others.  fp16 has no such rows.
template <int kElem, int kStream>
__device__ __forceinline__ float norm_scale(float squares, float eps) {
    if (kElem == 2 && kStream == 2) return 1.0f;
    return squares > 0x1p120f ? 0x1p-80f : squares < 0x1p-100f && eps < 0x1p-76f ? 0x1p100f : 1.0f;
}

// Sum over the T threads of a row; they all get it.  `at`: LDS of a wave's sum each, which nothing else uses until the next
// barrier but one.
template <int T>
__device__ __forceinline__ float over_row(float v, float* at) {
    v = row_sum<6>(v);
    if constexpr (T > 64) {
        if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = v;
        __syncthreads();
        v = at[0];
#pragma unroll
        for (int i = 1; i < T / 64; ++i) v += at[i];
    }
    return v;
}
template <int T>
__device__ __forceinline__ float most_of_row(float v, float* at) {
    v = row_max<6>(v);
    if constexpr (T > 64) {
        if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = v;
        __syncthreads();
        v = at[0];
#pragma unroll
        for (int i = 1; i < T / 64; ++i) v = fmaxf(v, at[i]);
    }
    return v;
}

template <int T>
constexpr int kRowsAtOnce = T == 64 ? 4 : 1;

// Workgroup: T threads a row, four rows where a wave takes one.
template <int kElem, int kStream, bool kQ8, int T, int K, bool kFar>
__global__ __launch_bounds__(T * kRowsAtOnce<T>) void norm_kernel(NormParams p) {
    __shared__ float sums[3][T / 64];
    const int t = threadIdx.x % T;
    const int row = blockIdx.x * kRowsAtOnce<T> + threadIdx.x / T;
    if (kRowsAtOnce<T> > 1 && row >= p.rows) return;  // a whole wave, and there are no barriers
    const long long b = row / p.N, n = row - (int)b * p.N;
    const char* x = p.x.data + (b * p.x.batch + n * p.x.token) * Io<kElem>::kBytes;
    const char* res = p.stream.data + (b * p.stream.batch + n * p.stream.token) * Io<kStream>::kBytes;
    char* sum = p.sum.data + (b * p.sum.batch + n * p.sum.token) * Io<kStream>::kBytes;
    char* out = p.out.data + (b * p.out.batch + n * p.out.token) * (kQ8 ? 1 : Io<kElem>::kBytes);

    int first[K], count[K];
    Eight<kElem, kFar> rx[K];
    Eight<kStream, kFar> rr[K];
    float s[K][8], w[K][8];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        first[k] = 8 * (k * T + t);
        count[k] = min(max(p.C - first[k], 0), 8);
        rx[k].load(x + (size_t)first[k] * Io<kElem>::kBytes, count[k]);
        if (p.stream.data) rr[k].load(res + (size_t)first[k] * Io<kStream>::kBytes, count[k]);
    }
#pragma unroll
    for (int k = 0; k < K; ++k) load_weights<kElem>(p, first[k], count[k], w[k]);
    float squares = 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        rx[k].get(s[k]);
        if (p.stream.data) {
            float r[8];
            rr[k].get(r);
#pragma unroll
            for (int j = 0; j < 8; ++j) s[k][j] += r[j];
            if (p.sum.data) Eight<kStream, kFar>::store(sum + (size_t)first[k] * Io<kStream>::kBytes, count[k], s[k]);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) squares = fmaf(s[k][j], s[k][j], squares);
    }
    squares = over_row<T>(squares, sums[0]);
    float eps = p.eps;
    const float by = norm_scale<kElem, kStream>(squares, eps);
    if (__builtin_expect(by != 1.0f, 0)) {  // the same for all of a row
        squares = 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                s[k][j] *= by;
                squares = fmaf(s[k][j], s[k][j], squares);
            }
        squares = over_row<T>(squares, sums[1]);
        eps = eps * by * by;
    }
    const float r = 1.0f / sqrtf(squares / (float)p.C + eps);
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j) s[k][j] *= r * w[k][j];
    if constexpr (!kQ8) {
#pragma unroll
        for (int k = 0; k < K; ++k) Eight<kElem, kFar>::store(out + (size_t)first[k] * Io<kElem>::kBytes, count[k], s[k]);
        return;
    }
    // the largest of a group: eight channels of a thread, 4, 8 or 16 neighbouring threads
    float most[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        most[k] = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) most[k] = fmaxf(most[k], j < count[k] ? fabsf(s[k][j]) : 0.0f);
    }
    int width = p.C;
    if (p.group) {
        width = p.group;
#pragma unroll
        for (int k = 0; k < K; ++k)
            most[k] = p.group == 32 ? row_max<2>(most[k]) : p.group == 64 ? row_max<3>(most[k]) : row_max<4>(most[k]);
    } else {
        float all = most[0];
#pragma unroll
        for (int k = 1; k < K; ++k) all = fmaxf(all, most[k]);
        all = most_of_row<T>(all, sums[2]);
#pragma unroll
        for (int k = 0; k < K; ++k) most[k] = all;
    }
    float* scales = p.scales + (size_t)row * (p.C / width);
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (count[k] == 0) continue;
        const float m = fmaxf(most[k], kLeast), scale = m / kE4m3Most, back = kE4m3Most / m;
        if (first[k] % width == 0) scales[first[k] / width] = scale;
        uint32_t q[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            q[i] = __builtin_amdgcn_cvt_pk_fp8_f32(s[k][4 * i] * back, s[k][4 * i + 1] * back, 0, false);
            q[i] = __builtin_amdgcn_cvt_pk_fp8_f32(s[k][4 * i + 2] * back, s[k][4 * i + 3] * back, q[i], true);
        }
        typedef u32x2 Anywhere __attribute__((aligned(1), may_alias));
        char* to = out + first[k];
        if (count[k] >= 8) {
            if (kFar) __builtin_nontemporal_store(u32x2{q[0], q[1]}, reinterpret_cast<Anywhere*>(to));
            else *reinterpret_cast<Anywhere*>(to) = u32x2{q[0], q[1]};
        } else {
#pragma unroll
            for (int j = 0; j < 7; ++j)
                if (j < count[k]) to[j] = (char)(q[j >> 2] >> (8 * (j & 3)));
        }
    }
}

// Backward.  Workgroup g takes rows g, g + groups, ... (four at once where a wave takes one) and keeps its sums for the
// weight's gradient in registers; they go to one row of `partial`, and norm_weight_kernel adds the rows up in order.
template <int kElem, int kStream, int T, int K, bool kFar>
__global__ __launch_bounds__(T * kRowsAtOnce<T>) void norm_backward_kernel(NormParams p) {
    constexpr int R = kRowsAtOnce<T>;
    __shared__ float sums[2][2][T / 64], again[2][T / 64];
    __shared__ float joined[R > 1 ? 8 * T * K : 1];
    const int t = threadIdx.x % T, wave = threadIdx.x / T;
    int first[K], count[K];
    float w[K][8], dw[K][8];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        first[k] = 8 * (k * T + t);
        count[k] = min(max(p.C - first[k], 0), 8);
        load_weights<kElem>(p, first[k], count[k], w[k]);
#pragma unroll
        for (int j = 0; j < 8; ++j) dw[k][j] = 0.0f;
    }
    int turn = 0;
    for (int row = blockIdx.x * R + wave; row < p.rows; row += p.groups * R, turn ^= 1) {
        const long long b = row / p.N, n = row - (int)b * p.N;
        const char* dy = p.x.data + (b * p.x.batch + n * p.x.token) * Io<kElem>::kBytes;
        const char* in = p.stream.data + (b * p.stream.batch + n * p.stream.token) * Io<kStream>::kBytes;
        const char* along = p.grad.data + (b * p.grad.batch + n * p.grad.token) * Io<kStream>::kBytes;
        Eight<kElem, kFar> ry[K];
        Eight<kStream, kFar> rh[K], ra[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            rh[k].load(in + (size_t)first[k] * Io<kStream>::kBytes, count[k]);
            ry[k].load(dy + (size_t)first[k] * Io<kElem>::kBytes, count[k]);
            if (p.grad.data) ra[k].load(along + (size_t)first[k] * Io<kStream>::kBytes, count[k]);
        }
        float h[K][8], u[K][8];
        auto both = [&](float& squares, float& dot) {
            squares = dot = 0.0f;
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    squares = fmaf(h[k][j], h[k][j], squares);
                    dot = fmaf(u[k][j] * w[k][j], h[k][j], dot);
                }
        };
#pragma unroll
        for (int k = 0; k < K; ++k) {
            rh[k].get(h[k]);
            ry[k].get(u[k]);
        }
        float squares, dot, eps = p.eps;
        both(squares, dot);
        squares = row_sum<6>(squares);
        dot = row_sum<6>(dot);
        if constexpr (T > 64) {  // two rows' sums may be under way: a wave can be a barrier ahead
            if ((threadIdx.x & 63) == 0) {
                sums[turn][0][threadIdx.x >> 6] = squares;
                sums[turn][1][threadIdx.x >> 6] = dot;
            }
            __syncthreads();
            squares = sums[turn][0][0];
            dot = sums[turn][1][0];
#pragma unroll
            for (int i = 1; i < T / 64; ++i) {
                squares += sums[turn][0][i];
                dot += sums[turn][1][i];
            }
        }
        const float by = norm_scale<kElem, kStream>(squares, eps);
        if (__builtin_expect(by != 1.0f, 0)) {  // the same for all of a row
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int j = 0; j < 8; ++j) h[k][j] *= by;
            both(squares, dot);
            squares = over_row<T>(squares, again[0]);
            dot = over_row<T>(dot, again[1]);
            eps = eps * by * by;
        }
        const float r = 1.0f / sqrtf(squares / (float)p.C + eps);
        const float mean = r * dot / (float)p.C;  // of w dy n
        const float whole = r * by;               // r is that of the scaled row
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float a[8];
            if (p.grad.data) ra[k].get(a);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float norm = h[k][j] * r;
                dw[k][j] = fmaf(u[k][j], norm, dw[k][j]);
                h[k][j] = whole * (u[k][j] * w[k][j] - norm * mean) + (p.grad.data ? a[j] : 0.0f);
            }
            if (p.out.data)
                Eight<kElem, kFar>::store(p.out.data + (b * p.out.batch + n * p.out.token + first[k]) * Io<kElem>::kBytes, count[k], h[k]);
            if (p.sum.data)
                Eight<kStream, kFar>::store(p.sum.data + (b * p.sum.batch + n * p.sum.token + first[k]) * Io<kStream>::kBytes, count[k], h[k]);
        }
    }
    if (!p.partial) return;
    float* to = p.partial + (size_t)blockIdx.x * p.C;
    if constexpr (R > 1) {
#pragma unroll 1
        for (int turn_of = 0; turn_of < R; ++turn_of) {
            if (wave == turn_of)
#pragma unroll
                for (int k = 0; k < K; ++k)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        float* at = &joined[(k * 8 + j) * T + t];
                        dw[k][j] += turn_of ? *at : 0.0f;
                        *at = dw[k][j];
                    }
            __syncthreads();
        }
        if (wave != R - 1) return;
    }
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < count[k]) to[first[k] + j] = dw[k][j];
}

// dw = sum of the rows of `partial`.  Workgroup = 32 columns x 32 row groups; each thread adds its rows in order, the groups
// are joined in a fixed tree.
// us of both kernels with 8 columns x 128 groups, 16 x 64, 32 x 32: 16384 rows of 2048 59 57 56, of 4096 104 100 99, 2048 of 1024 15
// 13.7 12.7, 4096 of 16384 116 110 107 (bf16).
constexpr int kNormColumns = 32, kNormGroups = 32;
template <int kElem>
__global__ __launch_bounds__(kNormColumns * kNormGroups) void norm_weight_kernel(NormParams p) {
    __shared__ float part[kNormGroups][kNormColumns + 1];
    const int c = threadIdx.x % kNormColumns, g = threadIdx.x / kNormColumns, col = blockIdx.x * kNormColumns + c;
    float sum = 0.0f;
    if (col < p.C)
#pragma unroll 8
        for (int r = g; r < p.groups; r += kNormGroups) sum += p.partial[(size_t)r * p.C + col];
    part[g][c] = sum;
    __syncthreads();
    for (int half = kNormGroups / 2; half > 0; half /= 2) {
        if (g < half) part[g][c] += part[g + half][c];
        __syncthreads();
    }
    if (g == 0 && col < p.C) {
        const float v = part[0][c];
        if (p.weight_f32) static_cast<float*>(p.weight_grad)[col] = v;
        else Io<kElem>::template store<1>(static_cast<char*>(p.weight_grad) + (size_t)col * Io<kElem>::kBytes, &v);
    }
}

int norm_rows_at_once(int C) { return C <= 512 ? 4 : 1; }

// About as many workgroups as the device holds at once, each of which ends with one row of sums.  us with half, these and twice as
// many: 16384 rows of 2048 63 57 65, 4094 of 1001 fp32 - 20.6 23.4, 16384 of 4096 - 100 106 (bf16).  Loading the next row while one
// is worked on gained nothing (54.8 and 55.5, 99.3 and 99.0).
int norm_groups(int rows, int C) {
    const int at_once = norm_rows_at_once(C);
    const long need = ((long)rows + at_once - 1) / at_once, most = C <= 2048 ? 1024 : C <= 4096 ? 512 : 256;
    return (int)(need < most ? need : most);
}

template <int kElem, int kStream, bool kQ8, int T, int K>
static void launch_norm_t(const NormParams& p, hipStream_t stream) {
    constexpr int R = kRowsAtOnce<T>;
    const dim3 grid((unsigned)((p.rows + (long long)R - 1) / R)), block(T * R);
    if (p.far) hipLaunchKernelGGL((norm_kernel<kElem, kStream, kQ8, T, K, true>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((norm_kernel<kElem, kStream, kQ8, T, K, false>), grid, block, 0, stream, p);
}
template <int kElem, int kStream, bool kQ8>
static void launch_norm_c(const NormParams& p, hipStream_t stream) {
    if (p.C <= 512) launch_norm_t<kElem, kStream, kQ8, 64, 1>(p, stream);
    else if (p.C <= 1024) launch_norm_t<kElem, kStream, kQ8, 128, 1>(p, stream);
    else if (p.C <= 2048) launch_norm_t<kElem, kStream, kQ8, 256, 1>(p, stream);
    else if (p.C <= 4096) launch_norm_t<kElem, kStream, kQ8, 512, 1>(p, stream);
    else if (p.C <= 8192) launch_norm_t<kElem, kStream, kQ8, 1024, 1>(p, stream);
    else launch_norm_t<kElem, kStream, kQ8, 1024, 2>(p, stream);
}
template <int kElem, int kStream>
static void launch_norm_q(const NormParams& p, bool q8, hipStream_t stream) {
    if (q8) launch_norm_c<kElem, kStream, true>(p, stream);
    else launch_norm_c<kElem, kStream, false>(p, stream);
}

hipError_t launch_norm(const NormParams& p, int elem, int stream_elem, bool q8, hipStream_t stream) {
    if (elem == 0) launch_norm_q<0, 0>(p, q8, stream);
    else if (elem == 1 && stream_elem == 0) launch_norm_q<1, 0>(p, q8, stream);
    else if (elem == 1) launch_norm_q<1, 1>(p, q8, stream);
    else if (stream_elem == 0) launch_norm_q<2, 0>(p, q8, stream);
    else launch_norm_q<2, 2>(p, q8, stream);
    return hipGetLastError();
}

template <int kElem, int kStream, int T, int K>
static void launch_norm_backward_t(const NormParams& p, hipStream_t stream) {
    const dim3 grid((unsigned)p.groups), block(T * kRowsAtOnce<T>);
    if (p.far) hipLaunchKernelGGL((norm_backward_kernel<kElem, kStream, T, K, true>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((norm_backward_kernel<kElem, kStream, T, K, false>), grid, block, 0, stream, p);
}
template <int kElem, int kStream>
static void launch_norm_backward_c(const NormParams& p, hipStream_t stream) {
    if (p.C <= 512) launch_norm_backward_t<kElem, kStream, 64, 1>(p, stream);
    else if (p.C <= 1024) launch_norm_backward_t<kElem, kStream, 128, 1>(p, stream);
    else if (p.C <= 2048) launch_norm_backward_t<kElem, kStream, 256, 1>(p, stream);
    else if (p.C <= 4096) launch_norm_backward_t<kElem, kStream, 512, 1>(p, stream);
    else if (p.C <= 8192) launch_norm_backward_t<kElem, kStream, 1024, 1>(p, stream);
    else launch_norm_backward_t<kElem, kStream, 1024, 2>(p, stream);
}

hipError_t launch_norm_backward(const NormParams& p, int elem, int stream_elem, hipStream_t stream) {
    if (elem == 0) launch_norm_backward_c<0, 0>(p, stream);
    else if (elem == 1 && stream_elem == 0) launch_norm_backward_c<1, 0>(p, stream);
    else if (elem == 1) launch_norm_backward_c<1, 1>(p, stream);
    else if (stream_elem == 0) launch_norm_backward_c<2, 0>(p, stream);
    else launch_norm_backward_c<2, 2>(p, stream);
    return hipGetLastError();
}

hipError_t launch_norm_weight(const NormParams& p, int elem, hipStream_t stream) {
    const dim3 grid((unsigned)((p.C + kNormColumns - 1) / kNormColumns)), block(kNormColumns * kNormGroups);
    if (elem == 0) hipLaunchKernelGGL((norm_weight_kernel<0>), grid, block, 0, stream, p);
    else if (elem == 1) hipLaunchKernelGGL((norm_weight_kernel<1>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((norm_weight_kernel<2>), grid, block, 0, stream, p);
    return hipGetLastError();
}

}  // namespace leet
