// The norm over all gradients of a model, and the gradients clipped to it.
//
//     norm = sqrt(sum of all squares),      out = g min(1, limit / norm)
//
// Bound by memory: the gradients are read for the norm and, once it is known, read again and written.  Two launches for up to 64
// tensors, whose addresses travel as kernel arguments; each workgroup of the second adds up the first one's sums by itself.  The
// second launch goes through the tensors from the last to the first, whose end the last-level cache still holds.  453 MB of bf16
// into buffers of their own: 80 and 153 us, 5.7 and 5.9 TB/s; twenty small tensors 5 and 8 us.
// Squares are added in fp64, which neither overflows nor loses the small ones, each workgroup's in an order of its own that
// does not depend on timing.
#include "leet_clip.hpp"
#include "leet_io.hpp"

namespace leet {

constexpr int kClipThreads = 256, kClipPieces = kClipTile / (8 * kClipThreads);  // pieces of eight elements

__device__ __forceinline__ double block_sum(double v, double* at) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = v;
    __syncthreads();
    v = at[0];
#pragma unroll
    for (int i = 1; i < kClipThreads / 64; ++i) v += at[i];
    return v;
}

// The tensor that a tile is of: the last one that begins at it or before it (empty ones begin where the next one does).
__device__ __forceinline__ int tensor_of(const ClipParams& p, int tile) {
    int lo = 0, hi = p.tensors;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (p.first[mid] <= tile) lo = mid;
        else hi = mid;
    }
    return lo;
}

// A tile's elements of one thread: pieces of eight, kClipThreads of them beside one another.
template <int kElem>
struct Tile {
    static constexpr int kBytes = Io<kElem>::kBytes, kWords = kElem == 0 ? 2 : 1;
    using Word = typename std::conditional<kElem == 0, u32x4, u32x4>::type;  // a dependent type, for an alignment that is one
    typedef Word Anywhere __attribute__((aligned(kBytes), may_alias));
    Word word[kClipPieces][kWords];

    static __device__ __forceinline__ int at(int i) { return 8 * (i * kClipThreads + threadIdx.x); }
    // all loads before any of them is looked at; zeros behind the tensor's end
    __device__ __forceinline__ void load(const char* p, int count) {
        if (count == kClipTile) {
#pragma unroll
            for (int i = 0; i < kClipPieces; ++i)
#pragma unroll
                for (int j = 0; j < kWords; ++j) word[i][j] = *(reinterpret_cast<const Anywhere*>(p + (size_t)at(i) * kBytes) + j);
            return;
        }
#pragma unroll
        for (int i = 0; i < kClipPieces; ++i) {
#pragma unroll
            for (int j = 0; j < kWords; ++j) word[i][j] = Word{0u, 0u, 0u, 0u};
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (at(i) + e < count) {
                    if constexpr (kElem == 0) word[i][e >> 2][e & 3] = reinterpret_cast<const uint32_t*>(p)[at(i) + e];
                    else word[i][0][e >> 1] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[at(i) + e] << (16 * (e & 1));
                }
        }
    }
    __device__ __forceinline__ float get(int i, int e) const {
        if constexpr (kElem == 0) return __builtin_bit_cast(float, (uint32_t)word[i][e >> 2][e & 3]);
        else return e & 1 ? Io<kElem>::hi(word[i][0][e >> 1]) : Io<kElem>::lo(word[i][0][e >> 1]);
    }
    __device__ __forceinline__ double squares() const {
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < kClipPieces; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const double v = get(i, e);
                sum = fma(v, v, sum);
            }
        return sum;
    }
    template <bool kFar>
    static __device__ __forceinline__ void put(char* p, Word w) {
        if (kFar) __builtin_nontemporal_store(w, reinterpret_cast<Anywhere*>(p));
        else *reinterpret_cast<Anywhere*>(p) = w;
    }
    template <bool kFar>
    __device__ __forceinline__ void store(char* p, int count, float first, float by) const {
#pragma unroll
        for (int i = 0; i < kClipPieces; ++i) {
            float f[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = get(i, e) * first * by;
            char* to = p + (size_t)at(i) * kBytes;
            if (at(i) + 8 <= count) {
                if constexpr (kElem == 0) {
                    put<kFar>(to, __builtin_bit_cast(Word, f32x4{f[0], f[1], f[2], f[3]}));
                    put<kFar>(to + 16, __builtin_bit_cast(Word, f32x4{f[4], f[5], f[6], f[7]}));
                } else {
                    put<kFar>(to, Word{Io<kElem>::pack2(f[0], f[1]), Io<kElem>::pack2(f[2], f[3]), Io<kElem>::pack2(f[4], f[5]),
                                       Io<kElem>::pack2(f[6], f[7])});
                }
            } else {
#pragma unroll
                for (int e = 0; e < 7; ++e)
                    if (at(i) + e < count) Io<kElem>::template store<1>(to + e * kBytes, &f[e]);
            }
        }
    }
};

// Where a tile lies: its tensor's first element of it, and how many it has.
struct TileOf {
    int tensor, count;
    long long begin;
    __device__ __forceinline__ TileOf(const ClipParams& p, int tile) {
        tensor = tensor_of(p, tile);
        begin = (long long)(tile - p.first[tensor]) * kClipTile;
        const long long rest = p.count[tensor] - begin;
        count = rest < kClipTile ? (int)rest : kClipTile;
    }
};

template <int kElem>
__device__ __forceinline__ double tile_squares(const ClipParams& p, const TileOf& t) {
    Tile<kElem> x;
    x.load(p.data[t.tensor] + t.begin * Io<kElem>::kBytes, t.count);
    return x.squares();
}
template <int kElem, bool kFar>
__device__ __forceinline__ void tile_times(const ClipParams& p, const TileOf& t, float first, float by) {
    Tile<kElem> x;
    x.load(p.data[t.tensor] + t.begin * Io<kElem>::kBytes, t.count);
    x.template store<kFar>(p.out[t.tensor] + t.begin * Io<kElem>::kBytes, t.count, first, by);
}

__global__ __launch_bounds__(kClipThreads) void clip_squares_kernel(ClipParams p) {
    __shared__ double sums[kClipThreads / 64];
    const int tiles = p.first[p.tensors];
    double sum = 0.0;
    for (int tile = blockIdx.x; tile < tiles; tile += kClipParts) {
        const TileOf t(p, tile);
        const int elem = p.elem[t.tensor];
        sum += elem == 0 ? tile_squares<0>(p, t) : elem == 1 ? tile_squares<1>(p, t) : tile_squares<2>(p, t);
    }
    sum = block_sum(sum, sums);
    if (threadIdx.x == 0) p.parts[blockIdx.x] = sum + (p.add ? p.parts[blockIdx.x] : 0.0);
}

// kFar: the tensors exceed the last-level cache, and what is written goes past it.  453 MB of bf16 clipped into buffers of their own:
// 264 -> 240 us, with tiles of 16384 elements instead of 8192 234.
template <bool kFar>
__global__ __launch_bounds__(kClipThreads) void clip_kernel(ClipParams p) {
    __shared__ double sums[kClipThreads / 64];
    double sum = 0.0;
    for (int i = threadIdx.x; i < kClipParts; i += kClipThreads) sum += p.parts[i];
    const double norm = sqrt(block_sum(sum, sums));
    if (p.norm && blockIdx.x == 0 && threadIdx.x == 0) *p.norm = (float)norm;
    // a norm that is not a finite number, or none at all, clips nothing
    const double factor = norm > (double)p.limit && norm < __builtin_inf() ? (double)p.limit / norm : 1.0;
    // in two steps, the first one exact, where it lies under fp32's normal range
    const float first = factor < 0x1p-126 ? 0x1p-100f : 1.0f, by = (float)(factor < 0x1p-126 ? factor * 0x1p100 : factor);
    const int tiles = p.first[p.tensors];
    for (int turn = blockIdx.x; turn < tiles; turn += gridDim.x) {
        const TileOf t(p, tiles - 1 - turn);
        if (factor == 1.0 && p.out[t.tensor] == p.data[t.tensor]) continue;
        const int elem = p.elem[t.tensor];
        if (elem == 0) tile_times<0, kFar>(p, t, first, by);
        else if (elem == 1) tile_times<1, kFar>(p, t, first, by);
        else tile_times<2, kFar>(p, t, first, by);
    }
}

hipError_t launch_clip_squares(const ClipParams& p, hipStream_t stream) {
    hipLaunchKernelGGL(clip_squares_kernel, dim3(kClipParts), dim3(kClipThreads), 0, stream, p);
    return hipGetLastError();
}

hipError_t launch_clip(const ClipParams& p, hipStream_t stream) {
    const int tiles = p.first[p.tensors];
    const dim3 grid(tiles < 1 ? 1 : tiles < 2048 ? tiles : 2048), block(kClipThreads);
    if (p.far) hipLaunchKernelGGL((clip_kernel<true>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((clip_kernel<false>), grid, block, 0, stream, p);
    return hipGetLastError();
}

}  // namespace leet
