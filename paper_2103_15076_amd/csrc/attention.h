// attention.h -- attention among packed sequences (the meshes of a mini-batch, one behind the other), forward and backward.
//
// Queries [Tq, Hq, D], keys and values [Tk, Hkv, D]; sequence b has the query rows q_off[b] .. q_off[b+1] and the key rows
// k_off[b] .. k_off[b+1] (lq and lk of them); Hq / Hkv = G heads of queries share a head of keys.
//   s_ij = scale q_i k_j over the keys j of i's own sequence, causal: those with j <= i + (lk - lq);
//   p = softmax_j(s),  out = p v,  lse = log sum_j exp s   (a query without keys: out = 0, lse = -inf)
//   delta = sum_d gout out,  ds = p (gout v^T - delta),  gv = p^T gout,  gq = scale ds k,  gk = scale ds^T q
// (gk, gv summed over the group's G heads).
//
// All products go through the matrix instructions, 32 x 32 tiles of 16 deep (binary32: eight 2-deep ones chained, which take
// an operand laid out alike).  Every kernel is arranged so that the product of a pair of operands comes out with its lanes
// along what the next product contracts over NOT: scores are made as K Q^T (a lane: one query, 16 of the tile's 32 keys) where
// the sum over keys follows, and as Q K^T (a lane: one key) where the sum over queries follows.  The probabilities then are
// the next product's operand as they stand, without a trip through LDS; which keys a lane holds is a permutation that the
// other operand, read transposed from LDS, shares.  Softmax statistics are a lane's own, but for one exchange between
// a wave's halves.
//
// A workgroup works on the rows of one group: row r of a sequence is query r / G, head r % G of the group, so K and V are read
// once for all heads that share them.  Tiles are found from the offsets on the device (Segments), so no lengths are needed on
// the host and a call can be recorded into a graph.  Sums over a long axis are split over workgroups where there are too few
// tiles to fill the chip, and joined in a fixed order.  No atomics: results do not depend on scheduling.
//
// Rounding: scores, statistics and all sums are binary32.  For 16-bit features the probabilities and ds are rounded to the
// features' type, as the matrix instructions take them: half a step each, relative, of terms of a sum whose result is rounded
// to the same type.  It costs: relative errors (root mean square) of 2.5e-3 for 1.7e-3 on causal bfloat16, 2.8e-4 for 2.1e-4 on
// binary16, which operands of twice as many bits (a second product for the lower half of each) would spare.  delta is taken from out as stored.
// binary16 has few exponents (a weight of one of a hundred thousand keys is below its normal range), so there the probabilities
// are carried times 2^15 and ds times a power of two that keeps a key's or query's largest within the range (Range).
#pragma once
#include <type_traits>

#include "feature_types.h"

#pragma clang fp contract(off)

namespace attn {

using feat::BLOCK;
using feat::Most;
using feat::Sum;
using feat::over_halves;

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

typedef float Acc __attribute__((ext_vector_type(16)));

template <typename T>
struct Types;
template <>
struct Types<feat::bf16> {
    typedef feat::bf16 Frag __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ Acc mfma(Frag a, Frag b, Acc c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Types<feat::f16> {
    typedef feat::f16 Frag __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ Acc mfma(Frag a, Frag b, Acc c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};
template <>
struct Types<float> {
    typedef float Frag __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ Acc mfma(Frag a, Frag b, Acc c) {
#pragma unroll
        for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
        return c;
    }
};
template <typename T>
using Frag = typename Types<T>::Frag;

typedef unsigned Quad __attribute__((ext_vector_type(4)));  // 16 bytes

// A caller's array of heads: element d of head h of row t is p[t * row + h * head + d].
template <typename T>
struct Heads {
    T* p;
    long long row, head;
};

// Rows of a group: row r is query r / G, head r % G.  The division by a multiplication (one too many at most for r < 2^31).
struct Group {
    int G;
    unsigned inv;  // ceil(2^32 / G); 0 for G = 1
    __device__ __forceinline__ int query(int r) const {
        if (inv == 0) return r;
        int t = (int)__umulhi((unsigned)r, inv);
        if (t * G > r) --t;
        return t;
    }
};
inline Group heads_per_group(int G) { return Group{G, G == 1 ? 0u : (unsigned)(((1ull << 32) + G - 1) / G)}; }

struct Offsets {
    const int* q;
    const int* k;
    int B, Tq, Tk;
};

// The rows of an axis (length T, `times` rows each) in tiles of SIZE: segment 0 is what lies in front of the first sequence,
// segments 1 .. B the sequences, segment B + 1 what lies behind the last.  Segment i's tiles are numbered from
// floor(start_i / SIZE) + i, which leaves each at least the tiles it needs, and the whole floor(T / SIZE) + B + 2 numbers.
struct Tile {
    int seq;           // sequence, or -1: rows of none
    int start, len;    // of the segment, queries or keys
    int first;         // first of the tile's rows, counted from the segment's first (`times` a query); less than 2^30 of them
    bool on;
};
inline long long tile_numbers(long long T, int times, int size, int B) { return T * times / size + B + 2; }
__device__ __forceinline__ int clipped(int x, int T) { return x < 0 ? 0 : (x > T ? T : x); }
template <int SIZE>
__device__ __forceinline__ Tile find_tile(const int* __restrict__ off, int B, int T, int times, long long number) {
    // the last segment whose numbers start at or below this one (their starts ascend): of 64 candidates spread over those left, one a
    // lane, until they are neighbours; up to 62 sequences in one step, 2^24 in four.  (Descending offsets give some segment.)
    const int lane = (int)threadIdx.x & 63;
    int seg = 0;
    for (int left = B + 2; left > 1;) {
        const int apart = (left + 63) >> 6, ahead = lane * apart;
        const bool in = ahead < left;
        const int i = in ? seg + ahead : 0;
        const int start = i == 0 ? 0 : clipped(off[i - 1], T);
        const int count = __popcll(__ballot(in && (long long)start * times / SIZE + i <= number));
        const int skip = count > 0 ? (count - 1) * apart : 0;
        seg += skip;
        left = left - skip < apart ? left - skip : apart;
    }
    Tile t;
    t.start = seg == 0 ? 0 : clipped(off[seg - 1], T);
    int end = seg == B + 1 ? T : clipped(off[seg], T);
    if (end < t.start) end = t.start;
    t.len = end - t.start;
    t.seq = seg >= 1 && seg <= B ? seg - 1 : -1;
    const long long first = (number - ((long long)t.start * times / SIZE + seg)) * SIZE;
    t.on = first >= 0 && first < (long long)t.len * times;  // (below 0: offsets that descend)
    t.first = t.on ? (int)first : 0;
    return t;
}
__device__ __forceinline__ void sequence_rows(const int* __restrict__ off, int seq, int T, int* start, int* len) {
    const int s = clipped(off[seq], T), e = clipped(off[seq + 1], T);
    *start = s;
    *len = e > s ? e - s : 0;
}

// ---- tiles in LDS ---------------------------------------------------------------------------------
//
// Rows of DP features in 16-byte chunks, without padding; the chunks of row r are permuted by an exclusive or, so that 16
// rows' same chunk (a fragment along the features) and 4 rows' 4 neighbouring chunks (a transposed one) fall to different
// banks.  A period of the banks is 16 chunks, whole rows or a part of one.
template <typename T, int DP>
struct Rows {
    static constexpr int V = 16 / (int)sizeof(T), CHUNKS = DP / V;
    static __device__ __forceinline__ int twist(int r) {
        if constexpr (CHUNKS >= 16) return ((r & 3) << 2) | ((r >> 2) & 3);
        else if constexpr (CHUNKS == 8) return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
        else return (r >> 2) & 3;
    }
    // chunk c of row r, in elements
    static __device__ __forceinline__ int at(int r, int c) { return (r * CHUNKS + (c ^ twist(r))) * V; }
    // features 16 step + 8 half .. + 7 of the row: an operand whose rows are the tile's, contracted over the features
    static __device__ __forceinline__ Frag<T> along(const T* tile, int r, int step, int half) {
        Frag<T> f;
        if constexpr (sizeof(T) == 2) {
            f = *reinterpret_cast<const Frag<T>*>(tile + at(r, 2 * step + half));
        } else {
            typedef float Four __attribute__((ext_vector_type(4)));
            const Four a = *reinterpret_cast<const Four*>(tile + at(r, 4 * step + 2 * half));
            const Four b = *reinterpret_cast<const Four*>(tile + at(r, 4 * step + 2 * half + 1));
            f = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
        }
        return f;
    }
    // the transposed operand: its row is feature d0 + lane % 32, its eight values are the tile's rows r0 + 4 half + {0 .. 3}
    // and r0 + 8 + 4 half + {0 .. 3}: those that a lane of a product holds (see above)
    static __device__ __forceinline__ Frag<T> across(const T* tile, int r0, int d0, int lane) {
        const int half = lane >> 5;
        if constexpr (sizeof(T) == 2) {
            // (a transposing load: 16 lanes read 4 rows of 16 features, lane i gets feature i of the four)
            typedef short Four __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) Four LdsFour;
            const int i = lane & 15, r = r0 + 4 * half + (i >> 2), d = d0 + (lane & 16) + 4 * (i & 3);
            T* p = const_cast<T*>(tile);
            const Four a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsFour*)(p + at(r, d >> 3) + (d & 4)));
            const Four b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsFour*)(p + at(r + 8, d >> 3) + (d & 4)));
            typedef short Eight __attribute__((ext_vector_type(8)));
            const Eight e = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
            return __builtin_bit_cast(Frag<T>, e);
        } else {
            const int d = d0 + (lane & 31);
            Frag<T> f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int r = r0 + 8 * (j >> 2) + 4 * half + (j & 3);
                f[j] = tile[at(r, d >> 2) + (d & 3)];
            }
            return f;
        }
    }
};

// What a workgroup's lanes carry of a tile of ROWS rows between memory and LDS.
template <typename T, int DP, int ROWS>
struct Staged {
    static constexpr int CHUNKS = Rows<T, DP>::CHUNKS, V = Rows<T, DP>::V, N = (ROWS * CHUNKS + BLOCK - 1) / BLOCK;
    static constexpr bool EVEN = ROWS * CHUNKS % BLOCK == 0;
    Quad q[N];
    // row(r): address of row r of the tile, of which the first `rows` (one at least) are there; the others, and features behind
    // the D-th, become 0.  Loads are not conditional (those of no row take the last's), so that all are in flight together.
    template <typename Row>
    __device__ __forceinline__ void load(int D, int rows, Row row) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int u = (int)threadIdx.x + i * BLOCK, r = u / CHUNKS, c = u % CHUNKS;
            q[i] = *reinterpret_cast<const Quad*>(row(r < rows ? r : rows - 1) + (c * V < D ? c * V : 0));
        }
        if (rows < ROWS || D < DP) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int u = (int)threadIdx.x + i * BLOCK, r = u / CHUNKS, c = u % CHUNKS;
                if (r >= rows || c * V >= D) q[i] = Quad{0, 0, 0, 0};
            }
        }
    }
    __device__ __forceinline__ void store(T* tile) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int u = (int)threadIdx.x + i * BLOCK, r = u / CHUNKS, c = u % CHUNKS;
            if (EVEN || r < ROWS) *reinterpret_cast<Quad*>(tile + Rows<T, DP>::at(r, c)) = q[i];
        }
    }
};

// Fragments of this lane's own row (lane % 32 of 32), contracted over the features, straight from memory.
template <typename T, int DP>
__device__ __forceinline__ void own_row(const T* p, int D, int half, Frag<T>* f) {
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) {
        const int d = 16 * s + 8 * half;
        Frag<T> v;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = (T)0.0f;
        if (p && d < D) {
            if constexpr (sizeof(T) == 2) {
                v = *reinterpret_cast<const Frag<T>*>(p + d);
            } else {
                typedef float Four __attribute__((ext_vector_type(4)));
                const Four a = *reinterpret_cast<const Four*>(p + d), b = *reinterpret_cast<const Four*>(p + d + 4);
                v = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
            }
        }
        f[s] = v;
    }
}

// The eight values of a product's lane that are the operand of step kk (16 of the 32 contracted over).
template <typename T>
__device__ __forceinline__ Frag<T> as_operand(const Acc& a, int kk) {
    Frag<T> f;
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = (T)a[8 * kk + j];
    return f;
}

// A lane's accumulators (feature 32 db + 8 (r / 4) + 4 half + r % 4 of its row) times f, to a row of D features.
template <typename T, int DP>
__device__ __forceinline__ void store_own_row(T* p, int D, int half, const Acc* acc, float f) {
#pragma unroll
    for (int db = 0; db < DP / 32; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int d = 32 * db + 8 * g + 4 * half;
            if (d < D) {
                typedef T Four __attribute__((ext_vector_type(4)));
                Four v;
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = (T)(acc[db][4 * g + i] * f);
                *reinterpret_cast<Four*>(p + d) = v;
            }
        }
}

// Exponent that probabilities are raised by (they are at most 1, but for rounding).
template <typename T>
constexpr float RAISE = std::is_same_v<T, feat::f16> ? 15.0f : 0.0f;

// The power of two that a lane carries ds by: lowered, and the lane's accumulators with it, when a value would leave binary16's
// range; nothing for the other types.  A lane's ds all belong to one key (or query), as its accumulators do, half of them in the
// lane of the other half: each key has a power of its own, and what another lane holds (nothing, where there is no key) is nothing to it.
// It settles within the first few tiles.
template <typename T, int DB>
struct Range {
    float by = std::is_same_v<T, feat::f16> ? 0x1p40f : 1.0f;
    __device__ __forceinline__ void fit(Acc& ds, Acc* acc) {
        if constexpr (std::is_same_v<T, feat::f16>) {
            float most = 0.0f;
#pragma unroll
            for (int r = 0; r < 16; ++r) most = fmaxf(most, fabsf(ds[r]));
            if (__ballot(most * by > 0x1p15f)) {
                most = over_halves<Most>(most);
                // most < 2^e: by 2^(15 - e) it stays below 2^15.  (Infinite: whatever it is carried by)
                const float to = most * by > 0x1p15f && most < INFINITY ? ldexpf(1.0f, 15 - min(ilogbf(most) + 1, 120)) : by;
                const float f = to / by;
#pragma unroll
                for (int db = 0; db < DB; ++db)
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[db][r] *= f;
                by = to;
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) ds[r] *= by;
        }
    }
    __device__ __forceinline__ float back() const { return std::is_same_v<T, feat::f16> ? 1.0f / by : 1.0f; }
};

// The row of a lane's accumulators that register r holds, less 4 half.
__device__ __forceinline__ constexpr int acc_row(int r) { return 8 * (r >> 2) + (r & 3); }

__device__ __forceinline__ Acc zeros() {
    Acc a;
#pragma unroll
    for (int r = 0; r < 16; ++r) a[r] = 0.0f;
    return a;
}

// ---- forward ----------------------------------------------------------------------------------------
//
// ROW_WAVES = 4: a workgroup takes 128 rows, 32 a wave, and all waves walk all keys; ROW_WAVES = 1: 32 rows, and the waves
// share out the keys of each tile (few rows: single tokens, short sequences), their statistics and sums joined at the end.
template <typename T, int DP, int ROW_WAVES>
struct ForwardShape {
    static constexpr int ROWS = 32 * ROW_WAVES, KEY_WAVES = 4 / ROW_WAVES;
    static constexpr int KEYS = ROW_WAVES == 4 ? (sizeof(T) == 2 ? 64 : 32) : 128;  // of a tile
    static constexpr int OWN = KEYS / KEY_WAVES;                                    // of them a wave's
    static constexpr int TILE = KEYS * DP;                                          // elements
    static constexpr int BUFFERS = 4 * TILE * (int)sizeof(T) <= 80 * 1024 ? 2 : 1;  // two workgroups a compute unit
    static constexpr int LDS = 2 * BUFFERS * TILE * (int)sizeof(T);
};

struct Scale {
    float log2;    // scale * log2(e): scores in units of a bit
    float plain;
};

// (Registers for two workgroups a compute unit: all fit but those of <16-bit, 128, 1>, where 5 go to memory.)
template <typename T, int DP, int ROW_WAVES>
__global__ __launch_bounds__(BLOCK, sizeof(T) == 2 || DP <= 64 ? 2 : 1) void forward_kernel(Heads<const T> q, Heads<const T> k, Heads<const T> v, Offsets off, int Hq,
                                                        int Hkv, Group group, int D, int causal, int clear, float scale2, Heads<T> out,
                                                        float* __restrict__ lse, float* __restrict__ part_out,
                                                        float* __restrict__ part_lse) {
    using S = ForwardShape<T, DP, ROW_WAVES>;
    constexpr int KB = S::OWN / 32, DB = DP / 32;
    __shared__ __attribute__((aligned(16))) char lds[S::LDS];
    __shared__ float stat[S::KEY_WAVES > 1 ? 2 : 1][4][32];
    const int G = group.G, kvh = blockIdx.y, split = blockIdx.z, splits = gridDim.z;
    const Tile t = find_tile<S::ROWS>(off.q, off.B, off.Tq, G, (long long)gridDim.x - 1 - blockIdx.x);
    if (!t.on || (t.seq < 0 && !clear)) return;
    const int wave = (int)threadIdx.x >> 6, lane = (int)threadIdx.x & 63, half = lane >> 5;
    const int row = t.first + (ROW_WAVES > 1 ? 32 * wave : 0) + (lane & 31);
    const bool row_on = row < t.len * G;
    const int token = row_on ? group.query(row) : 0, head = kvh * G + (row_on ? row - token * G : 0);
    const size_t at_q = (size_t)(t.start + token);

    int k_start = 0, lk = 0;
    if (t.seq >= 0) sequence_rows(off.k, t.seq, off.Tk, &k_start, &lk);
    const int shift = lk - t.len;
    int k_begin = 0, k_end = lk;
    if (causal) {  // keys that the tile's last token sees
        const int last = group.query(t.first + S::ROWS - 1);
        const int e = (last < t.len - 1 ? last : t.len - 1) + shift + 1;
        k_end = e < 0 ? 0 : (e < lk ? e : lk);
    }
    if (splits > 1) {
        const int chunk = ((lk + splits - 1) / splits + S::KEYS - 1) / S::KEYS * S::KEYS;
        const long long b = (long long)split * chunk, e = b + chunk;
        k_begin = b < k_end ? (int)b : k_end;
        k_end = e < k_end ? (int)e : k_end;
    }

    Frag<T> fq[DP / 16];
    own_row<T, DP>(row_on && k_begin < k_end ? q.p + at_q * q.row + head * q.head : nullptr, D, half, fq);
    Acc acc[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) acc[db] = zeros();
    float m = -INFINITY, l = 0.0f;

    Staged<T, DP, S::KEYS> sk, sv;
    const T* const kp = k.p + (size_t)k_start * k.row + (size_t)kvh * k.head;
    const T* const vp = v.p + (size_t)k_start * v.row + (size_t)kvh * v.head;
    auto fetch = [&](int j0) {
        sk.load(D, k_end - j0, [&](int r) { return kp + (size_t)(j0 + r) * k.row; });
        sv.load(D, k_end - j0, [&](int r) { return vp + (size_t)(j0 + r) * v.row; });
    };
    if (k_begin < k_end) fetch(k_begin);
    int buffer = 0;
    for (int j0 = k_begin; j0 < k_end; j0 += S::KEYS) {
        T* const tk = reinterpret_cast<T*>(lds) + buffer * 2 * S::TILE;
        T* const tv = tk + S::TILE;
        if (S::BUFFERS == 1) __syncthreads();
        else buffer ^= 1;
        sk.store(tk);
        sv.store(tv);
        __syncthreads();
        if (j0 + S::KEYS < k_end) fetch(j0 + S::KEYS);
        const int own = ROW_WAVES > 1 ? 0 : wave * S::OWN;
        if (S::KEY_WAVES > 1 && j0 + own >= k_end) continue;  // (barriers are met: the loop's own are at its head)
        Acc s[KB];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            s[kb] = zeros();
#pragma unroll
            for (int d = 0; d < DP / 16; ++d)
                s[kb] = Types<T>::mfma(Rows<T, DP>::along(tk, own + 32 * kb + (lane & 31), d, half), fq[d], s[kb]);
        }
        // keys that this lane's query does not see
        const int seen = causal ? (token + shift + 1 < k_end ? token + shift + 1 : k_end) : k_end;
        if (j0 + own + S::OWN > (causal ? group.query(t.first) + shift + 1 : k_end) || j0 + own + S::OWN > k_end) {
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (j0 + own + 32 * kb + acc_row(r) + 4 * half >= seen) s[kb][r] = -INFINITY;
        }
        float most = s[0][0];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r) most = fmaxf(most, s[kb][r]);
        most = over_halves<Most>(most);
        const float now = fmaxf(m, most), base = now == -INFINITY ? 0.0f : now, base2 = base * scale2;
        float keep = __builtin_amdgcn_exp2f(m * scale2 - base2), raised = base2 - RAISE<T>;
        // (2^(s scale2 - base2) is off by the rounding of base2, which all of a row's weights share: it cancels.  Of scores so large that it
        // could leave the exponents' range the difference is taken first.)
        if (__ballot(fabsf(base2) > 0x1p20f)) {
            keep = __builtin_amdgcn_exp2f((m - base) * scale2);
            raised = -RAISE<T>;
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[kb][r] -= base;
        }
        m = now;
        float sum = 0.0f;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float p = __builtin_amdgcn_exp2f(fmaf(s[kb][r], scale2, -raised));
                s[kb][r] = p;
                sum += p;
            }
        l = fmaf(l, keep, sum);
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[db][r] *= keep;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) {
                const Frag<T> p = as_operand<T>(s[kb], kk);
#pragma unroll
                for (int db = 0; db < DB; ++db)
                    acc[db] = Types<T>::mfma(Rows<T, DP>::across(tv, own + 32 * kb + 16 * kk, 32 * db, lane), p, acc[db]);
            }
    }
    l = over_halves<Sum>(l);
    m *= scale2;
    if constexpr (S::KEY_WAVES > 1) {
        // the waves' statistics, then their sums, each wave's in turn
        static_assert(32 * DP * 4 <= S::LDS, "the sums of a wave fit the tiles' place");
        if (half == 0) {
            stat[0][wave][lane] = m;
            stat[1][wave][lane] = l;
        }
        __syncthreads();
        float all = -INFINITY;
#pragma unroll
        for (int w = 0; w < 4; ++w) all = fmaxf(all, stat[0][w][lane & 31]);
        const float base = all == -INFINITY ? 0.0f : all;
        l = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) l = fmaf(stat[1][w][lane & 31], __builtin_amdgcn_exp2f(stat[0][w][lane & 31] - base), l);
        const float keep = __builtin_amdgcn_exp2f(m - base);
        m = all;
        // [register][lane]: neighbouring lanes, neighbouring words
        float* sums = reinterpret_cast<float*>(lds);
        for (int w = 3; w >= 1; --w) {
            if (wave == w) {
#pragma unroll
                for (int db = 0; db < DB; ++db)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        float x = acc[db][r] * keep;
                        if (w < 3) x += sums[(db * 16 + r) * 64 + lane];
                        sums[(db * 16 + r) * 64 + lane] = x;
                    }
            }
            __syncthreads();
        }
        if (wave != 0) return;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[db][r] = fmaf(acc[db][r], keep, sums[(db * 16 + r) * 64 + lane]);
    }
    if (!row_on) return;
    const bool some = !(l == 0.0f);  // (NaN is some)
    const float inv = some ? 1.0f / l : 0.0f;
    const float lse2 = some ? m + (log2f(l) - RAISE<T>) : -INFINITY;
    if (splits > 1) {
        const size_t at = ((size_t)split * Hq + head) * off.Tq + at_q;
        store_own_row<float, DP>(part_out + at * D, D, half, acc, inv);
        if (half == 0) part_lse[at] = lse2;
    } else {
        store_own_row<T, DP>(out.p + at_q * out.row + head * out.head, D, half, acc, inv);
        if (half == 0 && lse) lse[(size_t)head * off.Tq + at_q] = lse2 * LN2;
    }
}

// The splits' outputs joined: each has its share of the row's sum, 2^(lse2 - lse2 of all).  A row of D features to D / 4 lanes.
template <typename T>
__global__ __launch_bounds__(BLOCK) void join_kernel(const float* __restrict__ part_out, const float* __restrict__ part_lse, int splits,
                                                     Offsets off, int Hq, int D, int clear, Heads<T> out, float* __restrict__ lse) {
    const int packs = D / 4;
    const long long rows = (long long)off.Tq * Hq;
    for (long long i = (long long)blockIdx.x * BLOCK + threadIdx.x; i < rows * packs; i += (long long)gridDim.x * BLOCK) {
        const long long row = i / packs;
        const int d = (int)(i % packs) * 4, head = (int)(row / off.Tq), t = (int)(row % off.Tq);
        if (!clear && (t < clipped(off.q[0], off.Tq) || t >= clipped(off.q[off.B], off.Tq))) continue;  // (rows of no sequence stay)
        float m = -INFINITY;
        for (int s = 0; s < splits; ++s) m = fmaxf(m, part_lse[(size_t)s * rows + row]);
        const float base = m == -INFINITY ? 0.0f : m;
        float l = 0.0f, acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int s = 0; s < splits; ++s) {
            const float w = __builtin_amdgcn_exp2f(part_lse[(size_t)s * rows + row] - base);
            const float4 x = *reinterpret_cast<const float4*>(part_out + ((size_t)s * rows + row) * D + d);
            l += w;
            acc[0] = fmaf(w, x.x, acc[0]);
            acc[1] = fmaf(w, x.y, acc[1]);
            acc[2] = fmaf(w, x.z, acc[2]);
            acc[3] = fmaf(w, x.w, acc[3]);
        }
        const bool some = !(l == 0.0f);
        const float inv = some ? 1.0f / l : 0.0f;
        typedef T Four __attribute__((ext_vector_type(4)));
        Four v;
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = (T)(acc[k] * inv);
        *reinterpret_cast<Four*>(out.p + (size_t)t * out.row + (size_t)head * out.head + d) = v;
        if (d == 0 && lse) lse[row] = some ? (m + log2f(l)) * LN2 : -INFINITY;
    }
}

// ---- backward ---------------------------------------------------------------------------------------

// delta[head][t] = sum_d gout out.  16 lanes a row.
template <typename T>
__global__ __launch_bounds__(BLOCK) void delta_kernel(Heads<const T> gout, Heads<const T> out, int Tq, int Hq, int D,
                                                      float* __restrict__ delta) {
    for (long long row = ((long long)blockIdx.x * BLOCK + threadIdx.x) >> 4; row < (long long)Tq * Hq; row += (long long)gridDim.x * BLOCK >> 4) {
        const int t = (int)(row / Hq), head = (int)(row % Hq), d = ((int)threadIdx.x & 15) * 8;  // (row: t * Hq + head)
        float s = 0.0f;
        if (d < D) {
            const T* a = gout.p + (size_t)t * gout.row + (size_t)head * gout.head + d;
            const T* b = out.p + (size_t)t * out.row + (size_t)head * out.head + d;
#pragma unroll
            for (int c = 0; c < 8; c += 16 / (int)sizeof(T)) {
                float x[16 / sizeof(T)], y[16 / sizeof(T)];
                feat::load_pack(a + c, 8, x);
                feat::load_pack(b + c, 8, y);
#pragma unroll
                for (int j = 0; j < 16 / (int)sizeof(T); ++j) s = fmaf(x[j], y[j], s);
            }
        }
        s = feat::over_lanes<Sum, 16>(s);
        if ((threadIdx.x & 15) == 0) delta[(size_t)head * Tq + t] = s;
    }
}

// Gradients of the keys and values: a workgroup takes 128 keys, 32 a wave, and walks the rows (queries and heads of the group).
// Scores are made as Q K^T: a lane has one key, so p and ds are operands of the sums over rows as they stand.
template <typename T, int DP>
struct KeysShape {
    static constexpr int KEYS = 128, ROWS = 32;
    static constexpr int TILE = ROWS * DP;
    // 16-bit rows of 128: a lane's key and value, two accumulators and two products are far more than the 256 registers of two waves a
    // SIMD; with the values in LDS 10 (bfloat16) to 15 (float16) registers still go to memory, some of them in every turn.  All that one LDS
    // fragment feeds is one matrix instruction, and the kernel is bound by LDS: 1.92 of the 3.17 ms of causal 3 x 8 k, both passes.
    static constexpr bool VALUES_IN_LDS = sizeof(T) == 2 && DP == 128;
    static constexpr int BUFFERS = 4 * TILE * (int)sizeof(T) <= 80 * 1024 ? 2 : 1;
};
template <typename T, int DP>
__global__ __launch_bounds__(BLOCK, sizeof(T) == 2 || DP <= 64 ? 2 : 1) void backward_keys_kernel(Heads<const T> gout, Heads<const T> q, Heads<const T> k, Heads<const T> v,
                                                              const float* __restrict__ lse, const float* __restrict__ delta,
                                                              Offsets off, int Hq, int Hkv, Group group, int D, int causal, int clear, Scale scale,
                                                              Heads<T> gk, Heads<T> gv, float* __restrict__ part_k,
                                                              float* __restrict__ part_v) {
    using S = KeysShape<T, DP>;
    constexpr int DB = DP / 32;
    __shared__ __attribute__((aligned(16))) T lds[S::BUFFERS * 2 * S::TILE];
    __shared__ __attribute__((aligned(16))) float stat[S::BUFFERS][2][S::ROWS];
    __shared__ __attribute__((aligned(16))) T own_v[S::VALUES_IN_LDS ? S::KEYS * DP : 8];
    const int G = group.G, kvh = blockIdx.y, split = blockIdx.z, splits = gridDim.z;
    const Tile t = find_tile<S::KEYS>(off.k, off.B, off.Tk, 1, blockIdx.x);
    if (!t.on || (t.seq < 0 && !clear)) return;
    const int wave = (int)threadIdx.x >> 6, lane = (int)threadIdx.x & 63, half = lane >> 5;
    const int key = t.first + 32 * wave + (lane & 31);
    const bool key_on = key < t.len;

    int q_start = 0, lq = 0;
    if (t.seq >= 0) sequence_rows(off.q, t.seq, off.Tq, &q_start, &lq);
    const int shift = t.len - lq;
    int r_begin = 0, r_end = lq * G;
    if (causal) {  // rows that see the tile's first key, or a later one; the others (which may see nothing, and hold anything) are not read
        const long long first = ((long long)t.first - shift) * G;
        r_begin = first <= 0 ? 0 : (first < r_end ? (int)first : r_end);
    }
    if (splits > 1) {
        const int chunk = ((lq * G + splits - 1) / splits + S::ROWS - 1) / S::ROWS * S::ROWS;
        const long long b = (long long)split * chunk, e = b + chunk;
        if (b > r_begin) r_begin = b < r_end ? (int)b : r_end;
        if (e < r_end) r_end = (int)e;
    }

    Frag<T> fk[DP / 16], fv[DP / 16];
    const bool any = key_on && r_begin < r_end;
    own_row<T, DP>(any ? k.p + (size_t)(t.start + key) * k.row + (size_t)kvh * k.head : nullptr, D, half, fk);
    own_row<T, DP>(any ? v.p + (size_t)(t.start + key) * v.row + (size_t)kvh * v.head : nullptr, D, half, fv);
    if constexpr (S::VALUES_IN_LDS) {  // (read by the wave that writes them)
#pragma unroll
        for (int s = 0; s < DP / 16; ++s)
            *reinterpret_cast<Frag<T>*>(own_v + Rows<T, DP>::at(32 * wave + (lane & 31), 2 * s + half)) = fv[s];
    }
    Acc ak[DB], av[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) {
        ak[db] = zeros();
        av[db] = zeros();
    }

    Range<T, DB> range;

    Staged<T, DP, S::ROWS> sq, sg;
    float st = 0.0f;
    auto fetch = [&](int r0) {
        auto place = [&](int r, int* token, int* head) {
            const int row = r0 + r, i = group.query(row);
            *token = q_start + i;
            *head = kvh * G + row - i * G;
        };
        sq.load(D, r_end - r0, [&](int r) {
            int tk, hd;
            place(r, &tk, &hd);
            return q.p + (size_t)tk * q.row + (size_t)hd * q.head;
        });
        sg.load(D, r_end - r0, [&](int r) {
            int tk, hd;
            place(r, &tk, &hd);
            return gout.p + (size_t)tk * gout.row + (size_t)hd * gout.head;
        });
        if ((int)threadIdx.x < 2 * S::ROWS) {
            int tk, hd;
            place((int)threadIdx.x % S::ROWS, &tk, &hd);
            const bool on = r0 + (int)threadIdx.x % S::ROWS < r_end;
            const size_t at = (size_t)hd * off.Tq + tk;
            if ((int)threadIdx.x < S::ROWS) {
                // rows of no keys, and those behind the last, have p = 0
                st = on ? lse[at] * LOG2E - RAISE<T> : INFINITY;
                if (st == -INFINITY) st = INFINITY;
            } else {
                st = on ? delta[at] : 0.0f;
            }
        }
    };
    if (r_begin < r_end) fetch(r_begin);
    int buffer = 0;
    for (int r0 = r_begin; r0 < r_end; r0 += S::ROWS) {
        T* const tq = lds + buffer * 2 * S::TILE;
        T* const tg = tq + S::TILE;
        float(*const ts)[S::ROWS] = stat[buffer];
        if (S::BUFFERS == 1) __syncthreads();
        else buffer ^= 1;
        sq.store(tq);
        sg.store(tg);
        if ((int)threadIdx.x < 2 * S::ROWS) ts[(int)threadIdx.x / S::ROWS][(int)threadIdx.x % S::ROWS] = st;
        __syncthreads();
        if (r0 + S::ROWS < r_end) fetch(r0 + S::ROWS);
        Acc p = zeros(), ds = zeros();
#pragma unroll
        for (int d = 0; d < DP / 16; ++d) {
            p = Types<T>::mfma(Rows<T, DP>::along(tq, lane & 31, d, half), fk[d], p);
            const Frag<T> value = S::VALUES_IN_LDS ? Rows<T, DP>::along(own_v, 32 * wave + (lane & 31), d, half) : fv[d];
            ds = Types<T>::mfma(Rows<T, DP>::along(tg, lane & 31, d, half), value, ds);
        }
        const bool border = causal && t.first + S::KEYS - 1 > group.query(r0) + shift;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const float4 ls = *reinterpret_cast<const float4*>(&ts[0][8 * g + 4 * half]);
            const float4 dl = *reinterpret_cast<const float4*>(&ts[1][8 * g + 4 * half]);
            const float l4[4] = {ls.x, ls.y, ls.z, ls.w}, d4[4] = {dl.x, dl.y, dl.z, dl.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = 4 * g + i;
                p[r] = __builtin_amdgcn_exp2f(fmaf(p[r], scale.log2, -l4[i]));
                ds[r] = p[r] * (ds[r] - d4[i]);  // (raised as p is)
            }
        }
        if (border) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const bool hidden = key > group.query(r0 + acc_row(r) + 4 * half) + shift;
                p[r] = hidden ? 0.0f : p[r];
                ds[r] = hidden ? 0.0f : ds[r];
            }
        }
        range.fit(ds, ak);
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            const Frag<T> fp = as_operand<T>(p, kk), fd = as_operand<T>(ds, kk);
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                av[db] = Types<T>::mfma(Rows<T, DP>::across(tg, 16 * kk, 32 * db, lane), fp, av[db]);
                ak[db] = Types<T>::mfma(Rows<T, DP>::across(tq, 16 * kk, 32 * db, lane), fd, ak[db]);
            }
        }
    }
    if (!key_on) return;
    const size_t row = (size_t)(t.start + key);
    constexpr float lower = std::is_same_v<T, feat::f16> ? 0x1p-15f : 1.0f;  // 2^-RAISE
    const float of_k = scale.plain * (lower * range.back());
    if (splits > 1) {
        const size_t at = (((size_t)split * off.Tk + row) * Hkv + kvh) * D;
        store_own_row<float, DP>(part_k + at, D, half, ak, of_k);
        store_own_row<float, DP>(part_v + at, D, half, av, lower);
    } else {
        store_own_row<T, DP>(gk.p + row * gk.row + (size_t)kvh * gk.head, D, half, ak, of_k);
        store_own_row<T, DP>(gv.p + row * gv.row + (size_t)kvh * gv.head, D, half, av, lower);
    }
}

// Gradient of the queries: a workgroup takes 128 rows, 32 a wave, and walks the keys, scores as K Q^T as in the forward pass.
template <typename T, int DP>
struct QueriesShape {
    static constexpr int ROWS = 128, KEYS = 32;
    static constexpr int TILE = KEYS * DP;
    static constexpr int BUFFERS = 4 * TILE * (int)sizeof(T) <= 80 * 1024 ? 2 : 1;
};
template <typename T, int DP>
__global__ __launch_bounds__(BLOCK, sizeof(T) == 2 || DP <= 64 ? 2 : 1) void backward_queries_kernel(Heads<const T> gout, Heads<const T> q, Heads<const T> k,
                                                                 Heads<const T> v, const float* __restrict__ lse,
                                                                 const float* __restrict__ delta, Offsets off, int Hq, int Hkv, Group group, int D,
                                                                 int causal, int clear, Scale scale, Heads<T> gq,
                                                                 float* __restrict__ part_q) {
    using S = QueriesShape<T, DP>;
    constexpr int DB = DP / 32;
    __shared__ __attribute__((aligned(16))) T lds[S::BUFFERS * 2 * S::TILE];
    const int G = group.G, kvh = blockIdx.y, split = blockIdx.z, splits = gridDim.z;
    const Tile t = find_tile<S::ROWS>(off.q, off.B, off.Tq, G, (long long)gridDim.x - 1 - blockIdx.x);
    if (!t.on || (t.seq < 0 && !clear)) return;
    const int wave = (int)threadIdx.x >> 6, lane = (int)threadIdx.x & 63, half = lane >> 5;
    const int row = t.first + 32 * wave + (lane & 31);
    const bool row_on = row < t.len * G;
    const int token = row_on ? group.query(row) : 0, head = kvh * G + (row_on ? row - token * G : 0);
    const size_t at_q = (size_t)(t.start + token);

    int k_start = 0, lk = 0;
    if (t.seq >= 0) sequence_rows(off.k, t.seq, off.Tk, &k_start, &lk);
    const int shift = lk - t.len;
    int k_begin = 0, k_end = lk;
    if (causal) {
        const int last = group.query(t.first + S::ROWS - 1);
        const int e = (last < t.len - 1 ? last : t.len - 1) + shift + 1;
        k_end = e < 0 ? 0 : (e < lk ? e : lk);
    }
    if (splits > 1) {
        const int chunk = ((lk + splits - 1) / splits + S::KEYS - 1) / S::KEYS * S::KEYS;
        const long long b = (long long)split * chunk, e = b + chunk;
        k_begin = b < k_end ? (int)b : k_end;
        k_end = e < k_end ? (int)e : k_end;
    }

    const bool any = row_on && k_begin < k_end;
    Frag<T> fq[DP / 16], fg[DP / 16];
    own_row<T, DP>(any ? q.p + at_q * q.row + (size_t)head * q.head : nullptr, D, half, fq);
    own_row<T, DP>(any ? gout.p + at_q * gout.row + (size_t)head * gout.head : nullptr, D, half, fg);
    float ls = any ? lse[(size_t)head * off.Tq + at_q] * LOG2E : INFINITY;
    if (ls == -INFINITY) ls = INFINITY;
    const float dl = any ? delta[(size_t)head * off.Tq + at_q] : 0.0f;
    Acc acc[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) acc[db] = zeros();
    Range<T, DB> range;

    Staged<T, DP, S::KEYS> sk, sv;
    const T* const kp = k.p + (size_t)k_start * k.row + (size_t)kvh * k.head;
    const T* const vp = v.p + (size_t)k_start * v.row + (size_t)kvh * v.head;
    auto fetch = [&](int j0) {
        sk.load(D, k_end - j0, [&](int r) { return kp + (size_t)(j0 + r) * k.row; });
        sv.load(D, k_end - j0, [&](int r) { return vp + (size_t)(j0 + r) * v.row; });
    };
    if (k_begin < k_end) fetch(k_begin);
    int buffer = 0;
    for (int j0 = k_begin; j0 < k_end; j0 += S::KEYS) {
        T* const tk = lds + buffer * 2 * S::TILE;
        T* const tv = tk + S::TILE;
        if (S::BUFFERS == 1) __syncthreads();
        else buffer ^= 1;
        sk.store(tk);
        sv.store(tv);
        __syncthreads();
        if (j0 + S::KEYS < k_end) fetch(j0 + S::KEYS);
        Acc p = zeros(), ds = zeros();
#pragma unroll
        for (int d = 0; d < DP / 16; ++d) {
            p = Types<T>::mfma(Rows<T, DP>::along(tk, lane & 31, d, half), fq[d], p);
            ds = Types<T>::mfma(Rows<T, DP>::along(tv, lane & 31, d, half), fg[d], ds);
        }
        const int seen = causal ? (token + shift + 1 < k_end ? token + shift + 1 : k_end) : k_end;
        const bool border = j0 + S::KEYS > (causal ? group.query(t.first) + shift + 1 : k_end) || j0 + S::KEYS > k_end;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const float x = __builtin_amdgcn_exp2f(fmaf(p[r], scale.log2, -ls));
            ds[r] = x * (ds[r] - dl);
        }
        if (border) {
#pragma unroll
            for (int r = 0; r < 16; ++r) ds[r] = j0 + acc_row(r) + 4 * half >= seen ? 0.0f : ds[r];
        }
        range.fit(ds, &acc[0]);
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            const Frag<T> fd = as_operand<T>(ds, kk);
#pragma unroll
            for (int db = 0; db < DB; ++db) acc[db] = Types<T>::mfma(Rows<T, DP>::across(tk, 16 * kk, 32 * db, lane), fd, acc[db]);
        }
    }
    if (!row_on) return;
    const float f = scale.plain * range.back();
    if (splits > 1) store_own_row<float, DP>(part_q + (((size_t)split * off.Tq + at_q) * Hq + head) * D, D, half, acc, f);
    else store_own_row<T, DP>(gq.p + at_q * gq.row + (size_t)head * gq.head, D, half, acc, f);
}

// Splits' sums added up, in their order; part [splits][rows][H][D].
template <typename T>
__global__ __launch_bounds__(BLOCK) void sum_kernel(const float* __restrict__ part, int splits, const int* __restrict__ off, int B, int rows,
                                                    int H, int D, int clear, Heads<T> out) {
    const int packs = D / 4;
    const long long n = (long long)rows * H * packs;
    for (long long i = (long long)blockIdx.x * BLOCK + threadIdx.x; i < n; i += (long long)gridDim.x * BLOCK) {
        const int t = (int)(i / ((long long)H * packs)), u = (int)(i % ((long long)H * packs)), head = u / packs, d = u % packs * 4;
        if (!clear && (t < clipped(off[0], rows) || t >= clipped(off[B], rows))) continue;
        float a[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int s = 0; s < splits; ++s) {
            const float4 x = *reinterpret_cast<const float4*>(part + ((size_t)s * n + i) * 4);
            a[0] += x.x;
            a[1] += x.y;
            a[2] += x.z;
            a[3] += x.w;
        }
        typedef T Four __attribute__((ext_vector_type(4)));
        Four v;
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = (T)a[k];
        *reinterpret_cast<Four*>(out.p + (size_t)t * out.row + (size_t)head * out.head + d) = v;
    }
}

}  // namespace attn
