// gradients.h -- the norm of all gradients of a network together, and clipping by it.
//
//   norm = sqrt(sum over tensors and values of g^2),  c = min(1, max_norm / (norm + 1e-6)),  out = c g
//
// Bound by memory: every value is read for the norm and, the coefficient being known only then, read again and written.
// Two kernels: squares_kernel leaves a partial sum per workgroup, scale_kernel's workgroups each add all partials up (16 KB at
// most from the caches, in one fixed order, so all arrive at the same norm), and scale.  Squares are summed in 64 bits: no
// gradient's square leaves the range, and the sum's rounding does not depend on how many values there are.  The tensors'
// table travels with the launch, TENSORS of them at a time; launches of many tables leave more partials than a workgroup should add
// up for each 8192 values that it scales, and total_kernel makes one sum of them first.
#pragma once
#include "feature_types.h"

#pragma clang fp contract(off)

namespace grads {

using feat::BLOCK;
using feat::Chunk;
using feat::load_pack;
using feat::store_pack;

constexpr int TENSORS = 120;              // per launch: the table stays below the 4 KB of a launch's arguments
constexpr long long CHUNK_VALUES = 8192;  // values that a workgroup takes at a time
constexpr int MAX_PARTIALS = 2048;        // per launch: eight workgroups a compute unit; and those that scale_kernel adds up

struct Table {
    const void* in[TENSORS];
    void* out[TENSORS];
    unsigned long long size_type[TENSORS];  // values << 2 | type
    unsigned first[TENSORS + 1];            // first chunk of the tensor
    int count;
};
static_assert(sizeof(Table) <= 4000, "a launch's arguments");

// tensor that chunk i belongs to
__device__ __forceinline__ int tensor_of(const Table& t, unsigned i) {
    int lo = 0, hi = t.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (t.first[mid] <= i) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// Body(pointer, first value, values of it) for the packs of chunk i that fall to this lane, four at a time.
template <typename T, typename Body>
__device__ __forceinline__ void packs_of(long long first, long long n, Body body) {
    constexpr int V = Chunk<T>::N, STEP = 4 * BLOCK * V;
    const long long last = first + CHUNK_VALUES < n ? first + CHUNK_VALUES : n;
    for (long long p = first + (long long)threadIdx.x * V; p < last; p += STEP) body(p, last);
}

template <typename T>
__device__ __forceinline__ double squares_of(const T* __restrict__ g, long long first, long long n) {
    constexpr int V = Chunk<T>::N;
    double s0 = 0.0, s1 = 0.0;
    packs_of<T>(first, n, [&](long long p, long long last) {
        float v[4][V];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const long long q = p + (long long)u * BLOCK * V;
            const long long left = last - q;
            load_pack(g + q, left > V ? V : (int)(left > 0 ? left : 0), v[u]);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int k = 0; k < V; k += 2) {
                const double a = (double)v[u][k], b = (double)v[u][k + 1];
                s0 = fma(a, a, s0);
                s1 = fma(b, b, s1);
            }
    });
    return s0 + s1;
}

// Over all 256 lanes, in every lane.
__device__ __forceinline__ double block_sum(double x, double* slots) {
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) x += __shfl_xor(x, d, 64);
    if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = x;
    __syncthreads();
    return (slots[0] + slots[1]) + (slots[2] + slots[3]);
}

__global__ __launch_bounds__(BLOCK) void squares_kernel(Table t, double* __restrict__ partial) {
    __shared__ double slots[BLOCK / 64];
    double s = 0.0;
    for (unsigned i = blockIdx.x; i < t.first[t.count]; i += gridDim.x) {
        const int k = tensor_of(t, i);
        const long long n = (long long)(t.size_type[k] >> 2), at = (long long)(i - t.first[k]) * CHUNK_VALUES;
        switch (t.size_type[k] & 3) {
            case 0: s += squares_of((const feat::f32*)t.in[k], at, n); break;
            case 1: s += squares_of((const feat::bf16*)t.in[k], at, n); break;
            default: s += squares_of((const feat::f16*)t.in[k], at, n); break;
        }
    }
    s = block_sum(s, slots);
    if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

// The sum of all partials, in every lane.
__device__ __forceinline__ double sum_of(const double* __restrict__ partial, int partials, double* slots) {
    double s = 0.0;
    int i = threadIdx.x;
    for (; i + 3 * BLOCK < partials; i += 4 * BLOCK) {
        double v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = partial[i + k * BLOCK];
#pragma unroll
        for (int k = 0; k < 4; ++k) s += v[k];
    }
    for (; i < partials; i += BLOCK) s += partial[i];
    return block_sum(s, slots);
}

__global__ __launch_bounds__(BLOCK) void total_kernel(const double* __restrict__ partial, int partials, double* __restrict__ total) {
    __shared__ double slots[BLOCK / 64];
    const double s = sum_of(partial, partials, slots);
    if (threadIdx.x == 0) *total = s;
}

__global__ __launch_bounds__(BLOCK) void norm_kernel(const double* __restrict__ partial, int partials, float* __restrict__ norm) {
    __shared__ double slots[BLOCK / 64];
    const double n = sqrt(sum_of(partial, partials, slots));
    if (threadIdx.x == 0) *norm = (float)n;
}

template <typename T>
__device__ __forceinline__ void scale_chunk(const T* g, T* out, long long first, long long n, float c) {
    constexpr int V = Chunk<T>::N;
    packs_of<T>(first, n, [&](long long p, long long last) {
        float v[4][V];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const long long q = p + (long long)u * BLOCK * V;
            const long long left = last - q;
            load_pack(g + q, left > V ? V : (int)(left > 0 ? left : 0), v[u]);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const long long q = p + (long long)u * BLOCK * V;
            const long long left = last - q;
#pragma unroll
            for (int k = 0; k < V; ++k) v[u][k] *= c;
            store_pack(out + q, left > V ? V : (int)(left > 0 ? left : 0), v[u]);
        }
    });
}

// Where nothing is to be scaled and the gradients stay where they are there is nothing to do.  (c is NaN where the norm is, and
// so is everything then; an infinite norm gives c = 0: infinite gradients become NaN, the others 0.)
__global__ __launch_bounds__(BLOCK) void scale_kernel(Table t, const double* __restrict__ partial, int partials, double max_norm,
                                                      float* __restrict__ norm) {
    __shared__ double slots[BLOCK / 64];
    const double n = sqrt(sum_of(partial, partials, slots));
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)n;
    const double ratio = max_norm / (n + 1e-6);
    const float c = ratio >= 1.0 ? 1.0f : (float)ratio;
    const unsigned chunks = t.first[t.count];
    for (unsigned j = blockIdx.x; j < chunks; j += gridDim.x) {
        // (from the end: what the squares' pass has read last is still in the caches)
        const unsigned i = chunks - 1 - j;
        const int k = tensor_of(t, i);
        if (c == 1.0f && t.in[k] == t.out[k]) continue;
        const long long m = (long long)(t.size_type[k] >> 2), at = (long long)(i - t.first[k]) * CHUNK_VALUES;
        switch (t.size_type[k] & 3) {
            case 0: scale_chunk((const feat::f32*)t.in[k], (feat::f32*)t.out[k], at, m, c); break;
            case 1: scale_chunk((const feat::bf16*)t.in[k], (feat::bf16*)t.out[k], at, m, c); break;
            default: scale_chunk((const feat::f16*)t.in[k], (feat::f16*)t.out[k], at, m, c); break;
        }
    }
}

}  // namespace grads
