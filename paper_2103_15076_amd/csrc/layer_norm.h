// layer_norm.h -- layer norm over the rows of features [N, C], forward and backward.
//
//   mean = sum_c x / C,  rstd = 1 / sqrt(sum_c (x - mean)^2 / C + eps),  xh = (x - mean) rstd,  y = gamma xh + beta
//   with h = gamma gy:  gx = rstd (h - mean_c(h) - xh mean_c(h xh)),  ggamma = sum_n gy xh,  gbeta = sum_n gy
//
// Both passes are bound by memory (8 to 24 operations a value).  A row is read once and stays in registers: LANES lanes of a
// wave (or, for the widest that fit, a workgroup) share it, NP packs of 16 bytes a lane.  The mean is taken first and the
// squares of the differences then, from the registers: nothing cancels, whatever the mean.  The backward pass makes all
// gradients in one walk over gy and x: a lane sees the same columns of every row of its workgroup, so the columns' sums stay
// in registers, 64 rows a lane at most, and are joined in two fixed stages in 64 bits (a workgroup's rows side by side; then
// workgroups' partials by finish_kernel): no atomics, results do not depend on scheduling.
#pragma once
#include "feature_types.h"

#pragma clang fp contract(off)

namespace lnorm {

using feat::BLOCK;
using feat::Chunk;
using feat::Sum;
using feat::load_pack;
using feat::over_lanes;
using feat::store_pack;

constexpr int MAX_C = 8192;  // widest row that stays in registers

// Sum over the lanes that share a row; BLOCK of them go through LDS (two slots used in turn, so that one barrier a sum will do).
template <int LANES>
struct RowSum {
    float (*slots)[BLOCK / 64];
    int turn = 0;
    __device__ __forceinline__ float operator()(float x) {
        if constexpr (LANES <= 64) {
            return over_lanes<Sum, LANES>(x);
        } else {
            x = over_lanes<Sum, 64>(x);
            float* s = slots[turn];
            turn ^= 1;
            if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = x;
            __syncthreads();
            return (s[0] + s[1]) + (s[2] + s[3]);
        }
    }
};

// Rows of LANES lanes: how many a workgroup takes side by side.
template <int LANES>
constexpr int rows_per_block() {
    return BLOCK / LANES;
}
// ... and one behind the other before it uses the first, so that enough loads are in flight: where a lane has a pack or two.
template <int LANES, int NP>
constexpr int rows_in_flight() {
    return LANES > 64 ? 1 : NP == 1 ? 4 : NP == 2 ? 2 : 1;
}

template <typename T, int LANES, int NP>
__global__ __launch_bounds__(BLOCK) void forward_kernel(const T* __restrict__ x, long long N, int C,
                                                        const float* __restrict__ gamma, const float* __restrict__ beta, float eps,
                                                        T* __restrict__ y, float* __restrict__ mean_out,
                                                        float* __restrict__ rstd_out) {
    constexpr int V = Chunk<T>::N, U = rows_in_flight<LANES, NP>(), R = rows_per_block<LANES>();
    __shared__ float slots[2][BLOCK / 64];
    RowSum<LANES> row_sum{slots};
    const int lane = (int)threadIdx.x % LANES;
    const long long row0 = ((long long)blockIdx.x * U) * R + (int)threadIdx.x / LANES;
    const float inv_c = 1.0f / (float)C;
    float v[U][NP][V];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const long long n = row0 + (long long)u * R;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int c0 = (lane + i * LANES) * V;
            load_pack(x + n * C + c0, n < N ? C - c0 : 0, v[u][i]);
        }
    }
    float g[NP][V], b[NP][V];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int c0 = (lane + i * LANES) * V;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            g[i][k] = gamma && c0 + k < C ? gamma[c0 + k] : 1.0f;
            b[i][k] = beta && c0 + k < C ? beta[c0 + k] : 0.0f;
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const long long n = row0 + (long long)u * R;
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int k = 0; k < V; ++k) s += v[u][i][k];
        const float mean = row_sum(s) * inv_c;
        float q = 0.0f;
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const float d = (lane + i * LANES) * V + k < C ? v[u][i][k] - mean : 0.0f;
                v[u][i][k] = d;
                q = fmaf(d, d, q);
            }
        const float rstd = 1.0f / sqrtf(row_sum(q) * inv_c + eps);
        if (n >= N) continue;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int c0 = (lane + i * LANES) * V;
#pragma unroll
            for (int k = 0; k < V; ++k) v[u][i][k] = fmaf(v[u][i][k] * rstd, g[i][k], b[i][k]);
            store_pack(y + n * C + c0, C - c0, v[u][i]);
        }
        if (lane == 0) {
            if (mean_out) mean_out[n] = mean;
            if (rstd_out) rstd_out[n] = rstd;
        }
    }
}

// Rows wider than MAX_C: read three times, from the caches mostly.
template <typename T>
__global__ __launch_bounds__(BLOCK) void forward_wide_kernel(const T* __restrict__ x, int C, const float* __restrict__ gamma,
                                                             const float* __restrict__ beta, float eps, T* __restrict__ y,
                                                             float* __restrict__ mean_out, float* __restrict__ rstd_out) {
    __shared__ float slots[2][BLOCK / 64];
    RowSum<BLOCK> row_sum{slots};
    const long long n = blockIdx.x;
    const T* p = x + n * C;
    float s = 0.0f;
    for (unsigned c = threadIdx.x; c < (unsigned)C; c += BLOCK) s += (float)p[c];
    const float mean = row_sum(s) / (float)C;
    float q = 0.0f;
    for (unsigned c = threadIdx.x; c < (unsigned)C; c += BLOCK) {
        const float d = (float)p[c] - mean;
        q = fmaf(d, d, q);
    }
    const float rstd = 1.0f / sqrtf(row_sum(q) / (float)C + eps);
    for (unsigned c = threadIdx.x; c < (unsigned)C; c += BLOCK)
        y[n * C + c] = (T)fmaf(((float)p[c] - mean) * rstd, gamma ? gamma[c] : 1.0f, beta ? beta[c] : 0.0f);
    if (threadIdx.x == 0) {
        if (mean_out) mean_out[n] = mean;
        if (rstd_out) rstd_out[n] = rstd;
    }
}

// Rows chunk * blockIdx.x and on, `chunk` of them (a multiple of the rows in flight).  partial [gridDim.x][2][C]: the workgroup's
// sums of gy xh and of gy; null: not wanted.
template <typename T, int LANES, int NP>
__global__ __launch_bounds__(BLOCK) void backward_kernel(const T* __restrict__ gy, const T* __restrict__ x, long long N, int C,
                                                         const float* __restrict__ gamma, const float* __restrict__ mean_in,
                                                         const float* __restrict__ rstd_in, long long chunk,
                                                         T* __restrict__ gx, float* __restrict__ partial) {
    constexpr int V = Chunk<T>::N, U = rows_in_flight<LANES, NP>() > 2 ? 2 : rows_in_flight<LANES, NP>(), R = rows_per_block<LANES>();
    __shared__ float slots[2][BLOCK / 64];
    RowSum<LANES> row_sum{slots};
    const int lane = (int)threadIdx.x % LANES;
    const float inv_c = 1.0f / (float)C;
    float g[NP][V], sg[NP][V], sb[NP][V];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int c0 = (lane + i * LANES) * V;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            g[i][k] = gamma && c0 + k < C ? gamma[c0 + k] : 1.0f;
            sg[i][k] = 0.0f;
            sb[i][k] = 0.0f;
        }
    }
    const long long first = (long long)blockIdx.x * chunk, last = first + chunk < N ? first + chunk : N;
    for (long long base = first; base < last; base += (long long)U * R) {
        float a[U][NP][V], b[U][NP][V], mean[U], rstd[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long n = base + u * R + (int)threadIdx.x / LANES;
            const bool on = n < last;
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const int c0 = (lane + i * LANES) * V;
                load_pack(gy + n * C + c0, on ? C - c0 : 0, a[u][i]);
                load_pack(x + n * C + c0, on ? C - c0 : 0, b[u][i]);
            }
            mean[u] = on ? mean_in[n] : 0.0f;
            rstd[u] = on ? rstd_in[n] : 0.0f;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long n = base + u * R + (int)threadIdx.x / LANES;
            float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
            for (int i = 0; i < NP; ++i)
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    // (behind the row's end gy is 0, and xh is made 0: the mean is not)
                    const float xh = (lane + i * LANES) * V + k < C ? (b[u][i][k] - mean[u]) * rstd[u] : 0.0f;
                    sb[i][k] += a[u][i][k];
                    sg[i][k] = fmaf(a[u][i][k], xh, sg[i][k]);
                    const float h = a[u][i][k] * g[i][k];
                    a[u][i][k] = h;
                    b[u][i][k] = xh;
                    s1 += h;
                    s2 = fmaf(h, xh, s2);
                }
            if (!gx) continue;
            s1 = row_sum(s1) * inv_c;
            s2 = row_sum(s2) * inv_c;
            if (n >= last) continue;
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const int c0 = (lane + i * LANES) * V;
#pragma unroll
                for (int k = 0; k < V; ++k) a[u][i][k] = rstd[u] * (a[u][i][k] - s1 - b[u][i][k] * s2);
                store_pack(gx + n * C + c0, C - c0, a[u][i]);
            }
        }
    }
    if (!partial) return;
    // the workgroup's rows side by side: all in one wave's lanes first (those a multiple of LANES apart), then the waves
    __shared__ float sums[LANES > 64 ? 1 : (BLOCK / 64) * (LANES < 64 ? 64 : LANES) * NP * V];
    float* out = partial + (size_t)blockIdx.x * 2 * C;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        if constexpr (LANES > 64) {
#pragma unroll
            for (int i = 0; i < NP; ++i)
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    const int c = (lane + i * LANES) * V + k;
                    if (c < C) out[(size_t)which * C + c] = which ? sb[i][k] : sg[i][k];
                }
        } else {
            constexpr int COLS = LANES * NP * V;
            if (which) __syncthreads();
#pragma unroll
            for (int i = 0; i < NP; ++i)
#pragma unroll
                for (int k = 0; k < V; ++k)
                    sums[((int)threadIdx.x / LANES) * COLS + (lane + i * LANES) * V + k] = which ? sb[i][k] : sg[i][k];
            __syncthreads();
            for (int c = threadIdx.x; c < C; c += BLOCK) {
                double s = 0.0;
                for (int r = 0; r < R; ++r) s += (double)sums[r * COLS + c];
                out[(size_t)which * C + c] = (float)s;
            }
        }
    }
}

// Rows wider than MAX_C: the gradient of x row by row, the columns' sums by a kernel of their own (a lane a column).
template <typename T>
__global__ __launch_bounds__(BLOCK) void backward_wide_kernel(const T* __restrict__ gy, const T* __restrict__ x, int C,
                                                              const float* __restrict__ gamma, const float* __restrict__ mean_in,
                                                              const float* __restrict__ rstd_in, T* __restrict__ gx) {
    __shared__ float slots[2][BLOCK / 64];
    RowSum<BLOCK> row_sum{slots};
    const size_t at = (size_t)blockIdx.x * C;
    const float mean = mean_in[blockIdx.x], rstd = rstd_in[blockIdx.x];
    float s1 = 0.0f, s2 = 0.0f;
    for (unsigned c = threadIdx.x; c < (unsigned)C; c += BLOCK) {
        const float h = (float)gy[at + c] * (gamma ? gamma[c] : 1.0f);
        s1 += h;
        s2 = fmaf(h, ((float)x[at + c] - mean) * rstd, s2);
    }
    s1 = row_sum(s1) / (float)C;
    s2 = row_sum(s2) / (float)C;
    for (unsigned c = threadIdx.x; c < (unsigned)C; c += BLOCK) {
        const float h = (float)gy[at + c] * (gamma ? gamma[c] : 1.0f);
        gx[at + c] = (T)(rstd * (h - s1 - ((float)x[at + c] - mean) * rstd * s2));
    }
}
template <typename T>
__global__ __launch_bounds__(BLOCK) void columns_wide_kernel(const T* __restrict__ gy, const T* __restrict__ x, long long N, int C,
                                                             const float* __restrict__ mean_in, const float* __restrict__ rstd_in,
                                                             long long chunk, float* __restrict__ partial) {
    const unsigned c = blockIdx.x * BLOCK + threadIdx.x;
    if (c >= (unsigned)C) return;
    const long long first = (long long)blockIdx.y * chunk, last = first + chunk < N ? first + chunk : N;
    float sg = 0.0f, sb = 0.0f;
    for (long long n = first; n < last; ++n) {
        const float g = (float)gy[n * C + c];
        sg = fmaf(g, ((float)x[n * C + c] - mean_in[n]) * rstd_in[n], sg);
        sb += g;
    }
    partial[((size_t)blockIdx.y * 2 + 0) * C + c] = sg;
    partial[((size_t)blockIdx.y * 2 + 1) * C + c] = sb;
}

// Columns of the workgroups' partials [groups][2 C] added up: 16 columns a workgroup, 16 lanes a column, each every 16th group in
// turn, then a tree.  Sums are in 64 bits, as those of a workgroup's rows side by side are; in binary32 a lane adds up 64 rows at most (of
// rows wider than MAX_C a 65535th of all, where that is more).
constexpr int FINISH_COLS = 16;
__global__ __launch_bounds__(BLOCK) void finish_kernel(const float* __restrict__ partial, int groups, int C,
                                                       float* __restrict__ ggamma, float* __restrict__ gbeta) {
    constexpr int PARTS = BLOCK / FINISH_COLS;
    __shared__ double sums[PARTS][FINISH_COLS];
    const int mine = (int)threadIdx.x % FINISH_COLS, part = (int)threadIdx.x / FINISH_COLS;
    const long long cols = 2ll * C;
    for (long long first = (long long)blockIdx.x * FINISH_COLS; first < cols; first += (long long)gridDim.x * FINISH_COLS) {
        const long long col = first + mine;
        double s = 0.0;
        if (col < cols) {
            int g = part;
            for (; g + 7 * PARTS < groups; g += 8 * PARTS) {
                float v[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = partial[(g + k * PARTS) * cols + col];
#pragma unroll
                for (int k = 0; k < 8; ++k) s += (double)v[k];
            }
            for (; g < groups; g += PARTS) s += (double)partial[g * cols + col];
        }
        sums[part][mine] = s;
        __syncthreads();
        if (part == 0 && col < cols) {
            for (int k = 1; k < PARTS; ++k) s += sums[k][mine];
            float* out = col < C ? ggamma : gbeta;
            if (out) out[col < C ? col : col - C] = (float)s;
        }
        __syncthreads();
    }
}

}  // namespace lnorm
