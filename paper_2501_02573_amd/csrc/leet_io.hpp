// Loads and stores of fp32, bf16 and fp16 elements as fp32 values, for the kernels that are bound by them.
#pragma once

#include <type_traits>

#include "leet_common.hpp"

namespace leet {

// kElem: 0 = fp32, 1 = bf16, 2 = fp16.  Stores round to nearest even.
template <int kElem>
struct Io {
    static constexpr int kBytes = kElem == 0 ? 4 : 2;

    static __device__ __forceinline__ float lo(uint32_t word) { return kElem == 1 ? ElemBf16::lo(word) : ElemF16::lo(word); }
    static __device__ __forceinline__ float hi(uint32_t word) { return kElem == 1 ? ElemBf16::hi(word) : ElemF16::hi(word); }
    static __device__ __forceinline__ uint32_t pack2(float a, float b) {
        return kElem == 1 ? ElemBf16::pack2(a, b) : ElemF16::pack2(a, b);
    }

    // One or two adjacent elements as they lie in memory, at any address that suits one (the hardware takes words at any
    // address), so that many can be under way before any is looked at.
    template <int V>
    struct Raw {
        static_assert(V == 1 || V == 2, "one or two elements");
        typedef float Pair __attribute__((ext_vector_type(2)));
        using Word = typename std::conditional<kElem == 0, typename std::conditional<V == 1, float, Pair>::type,
                                               typename std::conditional<V == 1, uint16_t, uint32_t>::type>::type;
        typedef Word Anywhere __attribute__((aligned(kElem == 0 ? 4 : 2), may_alias));
        Word word;

        __device__ __forceinline__ void load(const char* p) { word = *reinterpret_cast<const Anywhere*>(p); }
        __device__ __forceinline__ void get(float* f) const {
            if constexpr (kElem == 0 && V == 1) f[0] = word;
            else if constexpr (kElem == 0) { f[0] = word[0]; f[1] = word[1]; }
            else {
                f[0] = lo(word);
                if constexpr (V == 2) f[1] = hi(word);
            }
        }
        __device__ __forceinline__ void set(const float* f) {
            if constexpr (kElem == 0 && V == 1) word = f[0];
            else if constexpr (kElem == 0) word = Word{f[0], f[1]};
            else if constexpr (V == 1) word = (uint16_t)pack2(f[0], 0.0f);
            else word = pack2(f[0], f[1]);
        }
        // with the nontemporal hint: for outputs that the library does not read again
        __device__ __forceinline__ void store(char* p) const { __builtin_nontemporal_store(word, reinterpret_cast<Anywhere*>(p)); }
    };

    // One or four adjacent elements at p (aligned to all of them)
    template <int V>
    static __device__ __forceinline__ void load(const char* p, float* f) {
        static_assert(V == 1 || V == 4, "one or four elements");
        if constexpr (kElem == 0 && V == 1) f[0] = *reinterpret_cast<const float*>(p);
        else if constexpr (kElem == 0) {
            const f32x4 x = *reinterpret_cast<const f32x4*>(p);
#pragma unroll
            for (int j = 0; j < 4; ++j) f[j] = x[j];
        } else if constexpr (V == 1) f[0] = lo(*reinterpret_cast<const uint16_t*>(p));
        else {
            const u32x2 x = *reinterpret_cast<const u32x2*>(p);
            f[0] = lo(x[0]); f[1] = hi(x[0]); f[2] = lo(x[1]); f[3] = hi(x[1]);
        }
    }

    template <int V>
    static __device__ __forceinline__ void store(char* p, const float* f) {
        static_assert(V == 1 || V == 4, "one or four elements");
        if constexpr (kElem == 0 && V == 1) *reinterpret_cast<float*>(p) = f[0];
        else if constexpr (kElem == 0) *reinterpret_cast<f32x4*>(p) = f32x4{f[0], f[1], f[2], f[3]};
        else if constexpr (V == 1) *reinterpret_cast<uint16_t*>(p) = (uint16_t)pack2(f[0], 0.0f);
        else *reinterpret_cast<u32x2*>(p) = u32x2{pack2(f[0], f[1]), pack2(f[2], f[3])};
    }
};

}  // namespace leet
