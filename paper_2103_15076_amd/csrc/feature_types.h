// feature_types.h -- what the operators on rows of features (layer_norm.h, attention.h, gradients.h) share: the types of
// features (binary32, bfloat16, binary16), packs of 16 bytes of them, and sums over lanes.
//
// Arithmetic is in binary32 whatever the features' type; a value is rounded to the features' type (to nearest even) once,
// where it is stored (and where it becomes an operand of a matrix instruction, attention.h).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#pragma clang fp contract(off)

namespace feat {

constexpr int BLOCK = 256;

using f32 = float;
using bf16 = __bf16;
using f16 = _Float16;

// 16 bytes of features, at any address that is a multiple of a feature's size (the hardware takes wide accesses there)
template <typename T>
struct Chunk {
    static constexpr int N = 16 / (int)sizeof(T);
};
template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Loose {
    T v[Chunk<T>::N];
};

// `left` of a pack's values (all, none or some of them) as binary32; the others read as 0.
template <typename T>
__device__ __forceinline__ void load_pack(const T* __restrict__ p, int left, float* __restrict__ out) {
    constexpr int N = Chunk<T>::N;
    if (left >= N) {
        const Loose<T> t = *reinterpret_cast<const Loose<T>*>(p);
#pragma unroll
        for (int k = 0; k < N; ++k) out[k] = (float)t.v[k];
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) out[k] = k < left ? (float)p[k] : 0.0f;
    }
}

template <typename T>
__device__ __forceinline__ void store_pack(T* __restrict__ p, int left, const float* __restrict__ in) {
    constexpr int N = Chunk<T>::N;
    if (left >= N) {
        Loose<T> t;
#pragma unroll
        for (int k = 0; k < N; ++k) t.v[k] = (T)in[k];
        *reinterpret_cast<Loose<T>*>(p) = t;
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (k < left) p[k] = (T)in[k];
    }
}

template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), CTRL, 0xF, 0xF, true));
}

struct Sum {
    static __device__ __forceinline__ float of(float a, float b) { return a + b; }
};
struct Most {
    static __device__ __forceinline__ float of(float a, float b) { return fmaxf(a, b); }
};

// x with the x of the lane 16 (in the other row of a pair) or 32 (in the other half) away, combined, in every lane
template <typename Op, bool HALVES>
__device__ __forceinline__ float swapped(float x) {
    const unsigned u = __builtin_bit_cast(unsigned, x);
    const auto r = HALVES ? __builtin_amdgcn_permlane32_swap(u, u, false, false) : __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const unsigned a = r[0], b = r[1];  // (by themselves: a bit cast of a vector's element takes the vector's first)
    return Op::of(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}

// Op over each group of LANES neighbouring lanes (a power of two), in every lane of the group; the order does not depend on
// anything but LANES.  Exchanges within a row of 16 lanes go through the data-parallel primitives, those between rows through
// the lane swaps: none through LDS.
template <typename Op, int LANES>
__device__ __forceinline__ float over_lanes(float x) {
    if constexpr (LANES >= 2) x = Op::of(x, dpp<0xB1>(x));   // lanes 1 0 3 2
    if constexpr (LANES >= 4) x = Op::of(x, dpp<0x4E>(x));   // lanes 2 3 0 1
    if constexpr (LANES >= 8) x = Op::of(x, dpp<0x141>(x));  // 7 .. 0 in each half row
    if constexpr (LANES >= 16) x = Op::of(x, dpp<0x140>(x)); // 15 .. 0 in each row
    if constexpr (LANES >= 32) x = swapped<Op, false>(x);
    if constexpr (LANES >= 64) x = swapped<Op, true>(x);
    return x;
}

// The two halves of a wave combined, in every lane.
template <typename Op>
__device__ __forceinline__ float over_halves(float x) {
    return swapped<Op, true>(x);
}

}  // namespace feat
