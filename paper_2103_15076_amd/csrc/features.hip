// features.hip -- entry points of the operators on rows of features that blocks of a network need beside the convolutions:
// layer norm (layer_norm.h), attention among packed sequences (attention.h), the norm of a network's gradients and clipping
// (gradients.h).  A translation unit of its own, beside picasso.hip.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include <algorithm>
#include <initializer_list>
#include <vector>

#include "../../include/picasso.h"
#include "attention.h"
#include "context.h"
#include "gradients.h"
#include "layer_norm.h"

#pragma clang fp contract(off)

namespace {

// The context's device is current while an operator queues its work, and the one before it afterwards.
struct OnDevice {
    int before = -1, now;
    hipError_t e;
    explicit OnDevice(int device) : now(device) {
        e = hipGetDevice(&before);
        if (e == hipSuccess && before != now) e = hipSetDevice(now);
    }
    ~OnDevice() {
        if (before >= 0 && before != now) (void)hipSetDevice(before);
    }
};

int failed(picasso_ctx* c, hipError_t e, const char* what) {
    char text[200];
    snprintf(text, sizeof text, "%s: %s", what, hipGetErrorString(e));
    picasso_note_hip_error(c, text);
    return PICASSO_ERR_HIP;
}
#define ON_DEVICE(c)                           \
    OnDevice on_device(picasso_device_of(c));  \
    if (on_device.e != hipSuccess) return failed(c, on_device.e, "selecting the context's device")
#define LAUNCHED(c)                                                      \
    do {                                                                 \
        const hipError_t e__ = hipGetLastError();                        \
        if (e__ != hipSuccess) return failed(c, e__, "a kernel's launch"); \
    } while (0)

bool known_type(int type) { return type == PICASSO_F32 || type == PICASSO_BF16 || type == PICASSO_F16; }
size_t size_of(int type) { return type == PICASSO_F32 ? 4 : 2; }
size_t up(size_t x) { return (x + 255) / 256 * 256; }
bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

// Memory that a call reads or writes, in bytes: `rows` times `heads` stretches of `width`, `row` and `head` apart.
struct Span {
    uintptr_t p;
    int64_t rows, row, heads, head, width;
    bool out;
    Span(const void* p_, int64_t rows_, int64_t row_, int64_t heads_, int64_t head_, int64_t width_, bool out_)
        : p((uintptr_t)p_), rows(rows_), row(row_), heads(heads_), head(head_), width(p_ ? width_ : 0), out(out_) {
        if (row == 0) rows = std::min<int64_t>(rows, 1);  // (broadcast)
        if (head == 0) heads = std::min<int64_t>(heads, 1);
        // stretches without a gap are one
        if (heads > 1 && head == width) width *= heads, heads = 1;
        if (rows > 1 && row == width) width *= rows, rows = 1;
        if (heads > 1 && head == width) width *= heads, heads = 1;
    }
    bool empty() const { return rows <= 0 || heads <= 0 || width <= 0; }
    int64_t extent() const { return empty() ? 0 : (rows - 1) * row + (heads - 1) * head + width; }
};
Span whole(const void* p, size_t bytes, bool out) { return Span(p, 1, 0, 1, 0, (int64_t)bytes, out); }

int64_t floor_div(int64_t x, int64_t y) { return x / y - (x % y < 0); }

// Whether a multiple of `row` by something from lo to hi puts x within (-below, above).
bool hits(int64_t x, int64_t row, int64_t lo, int64_t hi, int64_t below, int64_t above) {
    if (row == 0) return -below < x && x < above;
    return std::max(lo, floor_div(x - above, row) + 1) <= std::min(hi, floor_div(x + below - 1, row));
}

// Whether two spans have a byte in common.  Of arrays whose strides differ along an axis that both have it is not known: false.
bool meet(const Span& a, const Span& b) {
    if (a.empty() || b.empty() || a.p >= b.p + (uintptr_t)b.extent() || b.p >= a.p + (uintptr_t)a.extent()) return false;
    if ((a.rows > 1 && b.rows > 1 && a.row != b.row) || (a.heads > 1 && b.heads > 1 && a.head != b.head)) return false;
    const int64_t row = a.rows > 1 ? a.row : b.rows > 1 ? b.row : 0, head = a.heads > 1 ? a.head : b.heads > 1 ? b.head : 0, apart = (int64_t)(b.p - a.p);
    // parts of one projection, side by side in each row (what is passed as a rule)
    const int64_t wa = (a.heads - 1) * head + a.width, wb = (b.heads - 1) * head + b.width;
    if (row > 0) {
        const int64_t r = apart - floor_div(apart, row) * row;
        if (r >= wa && r + wb <= row) return false;
    }
    for (int64_t h = 1 - b.heads; h < a.heads; ++h)
        if (hits(apart - h * head, row, 1 - b.rows, a.rows - 1, b.width, a.width)) return true;
    return false;
}

// Whether two stretches of one array lie over each other.
bool folded(const Span& a) {
    if (a.empty()) return false;
    if (a.rows > 1 && a.row < a.width) return true;
    if (a.heads > 1 && a.head < a.width) return true;
    if (a.rows == 1 || a.heads == 1 || (a.heads - 1) * a.head + a.width <= a.row || (a.rows - 1) * a.row + a.width <= a.head) return false;
    for (int64_t h = 1; h < a.heads; ++h)
        if (hits(-h * a.head, a.row, 1 - a.rows, a.rows - 1, a.width, a.width)) return true;
    return false;
}

// What is written lies over nothing else that the call reads or writes.
bool apart(std::initializer_list<Span> all) {
    for (const Span* a = all.begin(); a != all.end(); ++a) {
        if (!a->out) continue;
        if (folded(*a)) return false;
        for (const Span* b = all.begin(); b != all.end(); ++b)
            if (a != b && (!b->out || a < b) && meet(*a, *b)) return false;
    }
    return true;
}

// Workgroups along an axis of a launch: fewer than 2^32 work items.  (More are not refused by the launch: it runs what is left of their
// number modulo 2^32.)
constexpr long long MAX_GROUPS = ((1ll << 32) - 1) / feat::BLOCK;
// ... of a kernel that walks `items` work items with the whole grid
unsigned groups_for(long long items) { return (unsigned)std::min((items + feat::BLOCK - 1) / feat::BLOCK, MAX_GROUPS); }

// CALL(T) for the features' type
#define FOR_TYPE(type, CALL)                           \
    do {                                               \
        if ((type) == PICASSO_F32) { CALL(feat::f32); }        \
        else if ((type) == PICASSO_BF16) { CALL(feat::bf16); } \
        else { CALL(feat::f16); }                      \
    } while (0)

// ---- layer norm -------------------------------------------------------------------------------------

// Lanes that share a row of C features, and packs a lane: as few lanes as hold it with a pack each, up to a wave; then up to
// four packs a lane; then a workgroup's lanes.
struct NormShape {
    int lanes, packs;
};
NormShape norm_shape(int C, int per_pack) {
    const int q = (int)((C + per_pack - 1ll) / per_pack);
    NormShape s{1, 1};
    while (s.lanes < 64 && s.lanes < q) s.lanes *= 2;
    if (q > 256) s.lanes = feat::BLOCK;
    while (s.lanes * s.packs < q) s.packs *= 2;
    return s;
}

#define NORM_SHAPES(T, s, CALL)                                                                                      \
    do {                                                                                                             \
        switch ((s).lanes) {                                                                                         \
            case 1: CALL(T, 1, 1); break;                                                                            \
            case 2: CALL(T, 2, 1); break;                                                                            \
            case 4: CALL(T, 4, 1); break;                                                                            \
            case 8: CALL(T, 8, 1); break;                                                                            \
            case 16: CALL(T, 16, 1); break;                                                                          \
            case 32: CALL(T, 32, 1); break;                                                                          \
            case 64:                                                                                                 \
                if ((s).packs == 1) CALL(T, 64, 1);                                                                  \
                else if ((s).packs == 2) CALL(T, 64, 2);                                                             \
                else CALL(T, 64, 4);                                                                                 \
                break;                                                                                               \
            default:                                                                                                 \
                if ((s).packs == 2) CALL(T, 256, 2);                                                                 \
                else if ((s).packs == 4) CALL(T, 256, 4);                                                            \
                else if constexpr (sizeof(T) == 4) CALL(T, 256, 8);                                                  \
        }                                                                                                            \
    } while (0)

// Workgroups of the backward pass, each with `chunk` rows and a partial sum of every column: 1024, fewer where each would have less
// than a few turns of rows, more where a lane would add up more than RUN rows in binary32 (the partials are joined in 64 bits).
// Partials are 8 bytes a channel for 64 rows or more that are read at 4 or 8 bytes and written at 2 or 4: 2 % of the traffic at most.
struct NormSplit {
    long long chunk;
    int groups;
};
constexpr long long RUN = 64;
NormSplit norm_split(long long N, int C, int type) {
    const bool wide = C > lnorm::MAX_C;  // (a lane a column: all of a workgroup's rows are its own)
    const long long beside = wide ? 1 : feat::BLOCK / norm_shape(C, 16 / (int)size_of(type)).lanes;
    const long long turn = wide ? RUN : 2 * beside;
    const long long groups = std::max(1ll, std::min(1024ll, (N + 2 * turn - 1) / (2 * turn)));
    const long long chunk = std::min(RUN * beside, std::max(1ll, ((N + groups - 1) / groups + turn - 1) / turn) * turn);
    // (columns_wide_kernel's workgroups along an axis that takes 65535)
    const long long least = wide ? (N + 65534) / 65535 : (N + MAX_GROUPS - 1) / MAX_GROUPS;
    const long long rows = std::max(chunk, (least + turn - 1) / turn * turn);
    return NormSplit{rows, (int)std::max(1ll, (N + rows - 1) / rows)};
}

// CALL(first row, rows) for launches of at most MAX_GROUPS workgroups of `per` rows each.
template <typename Call>
void by_rows(long long N, long long per, Call call) {
    for (long long at = 0; at < N; at += per * MAX_GROUPS) call(at, std::min(per * MAX_GROUPS, N - at));
}

template <typename T>
void launch_norm_forward(hipStream_t s, const T* x, long long N, int C, const float* gamma, const float* beta, float eps, T* y,
                         float* mean, float* rstd) {
    const auto from = [](float* p, long long at) { return p ? p + at : nullptr; };
    if (C > lnorm::MAX_C) {
        by_rows(N, 1, [&](long long at, long long n) {
            lnorm::forward_wide_kernel<T><<<(unsigned)n, feat::BLOCK, 0, s>>>(x + at * C, C, gamma, beta, eps, y + at * C, from(mean, at), from(rstd, at));
        });
        return;
    }
    const NormShape shape = norm_shape(C, feat::Chunk<T>::N);
#define PICASSO_CALL(T, L, P)                                                                                                   \
    do {                                                                                                                        \
        constexpr long long per = (long long)lnorm::rows_in_flight<L, P>() * lnorm::rows_per_block<L>();                         \
        by_rows(N, per, [&](long long at, long long n) {                                                                        \
            lnorm::forward_kernel<T, L, P><<<(unsigned)((n + per - 1) / per), feat::BLOCK, 0, s>>>(                              \
                x + at * C, n, C, gamma, beta, eps, y + at * C, from(mean, at), from(rstd, at));                                \
        });                                                                                                                     \
    } while (0)
    NORM_SHAPES(T, shape, PICASSO_CALL);
#undef PICASSO_CALL
}

template <typename T>
void launch_norm_backward(hipStream_t s, const T* gy, const T* x, long long N, int C, const float* gamma, const float* mean,
                          const float* rstd, T* gx, float* partial, const NormSplit& sp) {
    if (C > lnorm::MAX_C) {
        if (gx)
            by_rows(N, 1, [&](long long at, long long n) {
                lnorm::backward_wide_kernel<T><<<(unsigned)n, feat::BLOCK, 0, s>>>(gy + at * C, x + at * C, C, gamma, mean + at, rstd + at, gx + at * C);
            });
        if (partial)
            lnorm::columns_wide_kernel<T><<<dim3(groups_for(C), sp.groups), feat::BLOCK, 0, s>>>(gy, x, N, C, mean, rstd, sp.chunk, partial);
        return;
    }
    const NormShape shape = norm_shape(C, feat::Chunk<T>::N);
#define PICASSO_CALL(T, L, P) \
    lnorm::backward_kernel<T, L, P><<<sp.groups, feat::BLOCK, 0, s>>>(gy, x, N, C, gamma, mean, rstd, sp.chunk, gx, partial)
    NORM_SHAPES(T, shape, PICASSO_CALL);
#undef PICASSO_CALL
}

// ---- attention --------------------------------------------------------------------------------------

struct Attention {  // sizes of a call
    int type, B, Tq, Tk, Hq, Hkv, D;
    int G() const { return Hq / Hkv; }
    long long rows() const { return (long long)Tq * G(); }
};
bool valid(const Attention& a) {
    return known_type(a.type) && a.B >= 1 && a.B <= (1 << 24) && a.Tq >= 0 && a.Tk >= 0 && a.Tk <= (1 << 30) && a.Hq >= 1 && a.Hkv >= 1 &&
           a.Hq % a.Hkv == 0 && a.Hkv <= 65535 && a.D >= 8 && a.D <= 128 && a.D % 8 == 0 && a.rows() <= (1ll << 30) &&
           attn::tile_numbers(a.Tq, a.G(), 128, a.B) <= MAX_GROUPS && attn::tile_numbers(a.Tk, 1, 128, a.B) <= MAX_GROUPS;
}

// (the kernels take it times log2(e))
bool valid_scale(float scale) { return scale > 0.0f && std::isfinite(scale * attn::LOG2E); }

// Into how many parts an axis of `length` on average is split, where there are `groups` workgroups without: so that the chip has
// two a compute unit, parts of at least `least`.  Measured, backward pass alone, us with 1 / 2 / 4 / 8 splits of the rows: causal 3 x 8 k of 128
// features (2 by the rule) 3629 / 2804 / 2183 / 2131; 16 x 1536 of 32, float32 (1) 751 / 705 / 681 / 698; causal 1 x 4 k of 64 (8)
// 663 / 392 / 250 / 173; 4 x 1000 of 64, float16 (4) 86 / 76 / 80 / 87.  Where lengths or, causal, the work of tiles differ more parts than
// these would pay: the rule counts workgroups, not work.
int splits_for(long long groups, long long length, int least) {
    const long long wanted = (512 + groups - 1) / std::max(1ll, groups);
    return (int)std::max(1ll, std::min({wanted, length / least, 64ll}));
}

struct ForwardPlan {
    int row_waves, splits;
};
ForwardPlan forward_plan(const Attention& a) {
    const long long groups128 = (a.rows() / 128 + a.B) * a.Hkv, keys = a.Tk / a.B;
    ForwardPlan p;
    // Short sequences and single tokens: 32 rows a workgroup, whose waves share out the keys; and where there are too few groups of
    // 128 to fill the chip.  Measured, us with 32 | 128 rows: one mesh of 500, 4 heads of 32, float32 11.7 | 26.9, of 4 k 114 | 125; of 2 k, 8 heads of 64,
    // float32 108 | 118; bfloat16, 8 heads over 2 of 64, 500 9.1 | 12.0, 1 k 21.0 | 16.8, 4 k 97.5 | 60.7; 8 heads of 128, 64 meshes of 40
    // 26.6 | 12.1, 256 of 16 38.3 | 25.7.  So 32 rows are right for one mesh of up to about a thousand and in float32, and lose by up to
    // a factor of two and more among many short sequences and in 16 bits.
    p.row_waves = (a.rows() <= 48ll * a.B || groups128 < 256) && attn::tile_numbers(a.Tq, a.G(), 32, a.B) <= MAX_GROUPS ? 1 : 4;
    const long long groups = p.row_waves == 4 ? groups128 : (a.rows() / 32 + a.B) * a.Hkv;
    p.splits = splits_for(groups, keys, 256);
    return p;
}
struct BackwardPlan {
    int key_splits, query_splits;
};
BackwardPlan backward_plan(const Attention& a) {
    BackwardPlan p;
    p.key_splits = splits_for(((long long)a.Tk / 128 + a.B) * a.Hkv, a.rows() / a.B, 128);
    p.query_splits = splits_for((a.rows() / 128 + a.B) * a.Hkv, a.Tk / a.B, 128);
    return p;
}

size_t attention_forward_bytes(const Attention& a, const ForwardPlan& p) {
    if (p.splits == 1) return 0;
    return up((size_t)p.splits * a.Tq * a.Hq * a.D * 4) + up((size_t)p.splits * a.Tq * a.Hq * 4);
}
size_t attention_backward_bytes(const Attention& a, const BackwardPlan& p) {
    const size_t keys = p.key_splits == 1 ? 0 : 2 * up((size_t)p.key_splits * a.Tk * a.Hkv * a.D * 4);
    const size_t queries = p.query_splits == 1 ? 0 : up((size_t)p.query_splits * a.Tq * a.Hq * a.D * 4);
    return up((size_t)a.Tq * a.Hq * 4) + std::max(keys, queries);
}

// An array of heads as the kernels take it: 16-byte aligned rows and heads.
bool valid_heads(const picasso_heads* h, const Attention& a, int rows, int heads, bool output) {
    if (!h || (rows > 0 && !h->data)) return false;
    const long long each = (long long)(16 / size_of(a.type)), least = output ? a.D : 0;
    return aligned(h->data, 16) && h->row_stride >= least && h->head_stride >= least && h->row_stride % each == 0 && h->head_stride % each == 0 &&
           h->row_stride <= (1ll << 40) && h->head_stride <= (1ll << 40) &&
           (__int128)rows * h->row_stride + (__int128)heads * h->head_stride <= ((__int128)1 << 48);  // (no memory is larger)
}
Span span(const picasso_heads* h, const Attention& a, int rows, int heads, bool out) {
    const int64_t size = (int64_t)size_of(a.type);
    return Span(h->data, rows, h->row_stride * size, heads, h->head_stride * size, a.D * size, out);
}
template <typename T>
attn::Heads<T> heads(const picasso_heads* h) {
    return attn::Heads<T>{(T*)h->data, (long long)h->row_stride, (long long)h->head_stride};
}

// CALL(T, DP): features padded to 32, 64 or 128
#define FOR_WIDTH(T, D, CALL)                      \
    do {                                           \
        if ((D) <= 32) { CALL(T, 32); }            \
        else if ((D) <= 64) { CALL(T, 64); }       \
        else { CALL(T, 128); }                     \
    } while (0)

// ---- gradients --------------------------------------------------------------------------------------

// each(table, workgroups) for TENSORS tensors at a time (of sizes that `countable` has let pass).
template <typename Each>
void gradient_tables(int n, const void* const* in, void* const* out, const int64_t* sizes, const int32_t* types, Each each) {
    const int launches = std::max(1, (n + grads::TENSORS - 1) / grads::TENSORS);
    const int most = std::max(256, grads::MAX_PARTIALS / launches);
    for (int at = 0; at < n; at += grads::TENSORS) {
        grads::Table t;
        t.count = std::min(grads::TENSORS, n - at);
        unsigned long long chunks = 0;
        for (int k = 0; k < t.count; ++k) {
            t.in[k] = in ? in[at + k] : nullptr;
            t.out[k] = out ? out[at + k] : nullptr;
            t.size_type[k] = (unsigned long long)sizes[at + k] << 2 | (unsigned)(types ? types[at + k] : 0);
            t.first[k] = (unsigned)chunks;
            chunks += ((unsigned long long)sizes[at + k] + grads::CHUNK_VALUES - 1) / grads::CHUNK_VALUES;
        }
        t.first[t.count] = (unsigned)chunks;
        if (chunks) each(t, (int)std::min<unsigned long long>(chunks, most));
    }
}

// Sizes whose chunks a table can number: 2^43 values in all (2^30 chunks of 8192, and one more a tensor).
bool countable(int n, const int64_t* sizes) {
    int64_t all = 0;
    for (int k = 0; k < n; ++k) {
        if (sizes[k] < 0 || sizes[k] > (1ll << 43) - all) return false;
        all += sizes[k];
    }
    return true;
}

bool valid_gradients(int n, const void* const* in, const int64_t* sizes, const int32_t* types) {
    if (n < 0 || (n > 0 && (!in || !sizes || !types)) || !countable(n, sizes)) return false;
    for (int k = 0; k < n; ++k)
        if (!known_type(types[k]) || (sizes[k] > 0 && !in[k]) || !aligned(in[k], size_of(types[k])))
            return false;
    return true;
}

// What is written lies over nothing else: an output may be its own gradient, and nothing more (a tensor that is listed twice would be
// scaled twice, or once and a half); the norm and the workspace are no tensor's memory.  out: null, where tensors are only read.
int tensors_apart(int n, const void* const* in, void* const* out, const int64_t* sizes, const int32_t* types, const float* norm,
                  const void* ws, size_t ws_bytes) {
    struct Range {
        uintptr_t from, to;
        bool out;
    };
    std::vector<Range> r;
    try {
        r.reserve(2 * (size_t)n + 2);
    } catch (...) {
        return PICASSO_ERR_WORKSPACE;
    }
    const auto add = [&](const void* p, uintptr_t bytes, bool written) {
        if (p && bytes) r.push_back(Range{(uintptr_t)p, (uintptr_t)p + bytes, written});
    };
    // (outputs and gradients mostly ascend, each by themselves: sorted only where they do not)
    const auto ascends = [](const Range& a, const Range& b) { return a.from < b.from; };
    const auto sorted = [&](size_t first) {
        if (!std::is_sorted(r.begin() + first, r.end(), ascends)) std::sort(r.begin() + first, r.end(), ascends);
        std::inplace_merge(r.begin(), r.begin() + first, r.end(), ascends);
        return r.size();
    };
    for (int k = 0; out && k < n; ++k) add(out[k], (uintptr_t)sizes[k] * size_of(types[k]), true);
    const size_t outs = sorted(0);
    for (int k = 0; k < n; ++k)
        if (!out || out[k] != in[k]) add(in[k], (uintptr_t)sizes[k] * size_of(types[k]), false);
    const size_t tensors = sorted(outs);
    add(norm, sizeof(float), true);
    add(ws, ws_bytes, true);
    sorted(tensors);
    uintptr_t end_out = 0, end_any = 0;  // of those that start before
    for (const Range& x : r) {
        if (x.from < (x.out ? end_any : end_out)) return PICASSO_ERR_INVALID_ARG;
        end_any = std::max(end_any, x.to);
        if (x.out) end_out = std::max(end_out, x.to);
    }
    return PICASSO_OK;
}

// Partials of all tensors' squares in ws; how many.
int queue_squares(hipStream_t s, int n, const void* const* in, const int64_t* sizes, const int32_t* types, double* ws) {
    int partials = 0;
    gradient_tables(n, in, nullptr, sizes, types, [&](const grads::Table& t, int groups) {
        grads::squares_kernel<<<groups, feat::BLOCK, 0, s>>>(t, ws + partials);
        partials += groups;
    });
    return partials;
}

}  // namespace

extern "C" {

int picasso_layer_norm_forward(picasso_ctx* c, void* stream, int type, const void* d_x, int32_t N, int32_t C, const float* d_gamma,
                               const float* d_beta, float eps, void* d_y, float* d_mean, float* d_rstd) {
    if (!c || !known_type(type) || N < 0 || C < 1 || !(eps >= 0.0f) || !std::isfinite(eps) || (N > 0 && (!d_x || !d_y)))
        return PICASSO_ERR_INVALID_ARG;
    const size_t bytes = (size_t)N * C * size_of(type), stats = (size_t)N * 4, params = (size_t)C * 4;
    if (!aligned(d_x, size_of(type)) || !aligned(d_y, size_of(type)) ||
        !apart({whole(d_x, bytes, false), whole(d_gamma, params, false), whole(d_beta, params, false), whole(d_y, bytes, true),
                whole(d_mean, stats, true), whole(d_rstd, stats, true)}))
        return PICASSO_ERR_INVALID_ARG;
    if (N == 0) return PICASSO_OK;
    hipStream_t s = (hipStream_t)stream;
    ON_DEVICE(c);
#define PICASSO_CALL(T) launch_norm_forward<T>(s, (const T*)d_x, N, C, d_gamma, d_beta, eps, (T*)d_y, d_mean, d_rstd)
    FOR_TYPE(type, PICASSO_CALL);
#undef PICASSO_CALL
    LAUNCHED(c);
    return PICASSO_OK;
}

size_t picasso_layer_norm_workspace_bytes(int type, int32_t N, int32_t C) {
    if (!known_type(type) || N < 0 || C < 1) return 0;
    return (size_t)norm_split(N, C, type).groups * 2 * C * sizeof(float);
}

int picasso_layer_norm_backward(picasso_ctx* c, void* stream, int type, const void* d_gy, const void* d_x, int32_t N, int32_t C,
                                const float* d_gamma, const float* d_mean, const float* d_rstd, void* d_gx, float* d_ggamma,
                                float* d_gbeta, void* d_workspace, size_t workspace_bytes) {
    if (!c || !known_type(type) || N < 0 || C < 1 || (N > 0 && (!d_gy || !d_x || !d_mean || !d_rstd)) || (!d_gx && !d_ggamma && !d_gbeta))
        return PICASSO_ERR_INVALID_ARG;
    if (!aligned(d_gy, size_of(type)) || !aligned(d_x, size_of(type)) || !aligned(d_gx, size_of(type))) return PICASSO_ERR_INVALID_ARG;
    const bool sums = d_ggamma || d_gbeta;
    const size_t bytes = (size_t)N * C * size_of(type), stats = (size_t)N * 4, params = (size_t)C * 4,
                 need = sums ? picasso_layer_norm_workspace_bytes(type, N, C) : 0;
    if (!apart({whole(d_gy, bytes, false), whole(d_x, bytes, false), whole(d_gamma, params, false), whole(d_mean, stats, false),
                whole(d_rstd, stats, false), whole(d_gx, bytes, true), whole(d_ggamma, params, true), whole(d_gbeta, params, true),
                whole(d_workspace, std::min(need, workspace_bytes), true)}))
        return PICASSO_ERR_INVALID_ARG;
    if (sums && (!d_workspace || workspace_bytes < need)) return PICASSO_ERR_WORKSPACE;
    if (N == 0 && !sums) return PICASSO_OK;
    hipStream_t s = (hipStream_t)stream;
    ON_DEVICE(c);
    const NormSplit sp = norm_split(N, C, type);
    float* partial = sums ? (float*)d_workspace : nullptr;
#define PICASSO_CALL(T) \
    launch_norm_backward<T>(s, (const T*)d_gy, (const T*)d_x, N, C, d_gamma, d_mean, d_rstd, (T*)d_gx, partial, sp)
    FOR_TYPE(type, PICASSO_CALL);
#undef PICASSO_CALL
    if (sums)
        lnorm::finish_kernel<<<groups_for(2ll * C * (feat::BLOCK / lnorm::FINISH_COLS)), feat::BLOCK, 0, s>>>(partial, sp.groups, C, d_ggamma, d_gbeta);
    LAUNCHED(c);
    return PICASSO_OK;
}

size_t picasso_attention_workspace_bytes(int type, int32_t B, int32_t Tq, int32_t Tk, int32_t Hq, int32_t Hkv, int32_t D, int backward) {
    const Attention a{type, B, Tq, Tk, Hq, Hkv, D};
    if (!valid(a)) return 0;
    return backward ? attention_backward_bytes(a, backward_plan(a)) : attention_forward_bytes(a, forward_plan(a));
}

int picasso_attention_forward(picasso_ctx* c, void* stream, int type, const picasso_heads* q, const picasso_heads* k, const picasso_heads* v,
                              const int32_t* d_q_offsets, const int32_t* d_k_offsets, int32_t B, int32_t Tq, int32_t Tk, int32_t Hq,
                              int32_t Hkv, int32_t D, int causal, float scale, int clear_outside, const picasso_heads* out, float* d_lse,
                              void* d_workspace, size_t workspace_bytes) {
    const Attention a{type, B, Tq, Tk, Hq, Hkv, D};
    if (!c || !valid(a) || !valid_heads(q, a, Tq, Hq, false) || !valid_heads(k, a, Tk, Hkv, false) || !valid_heads(v, a, Tk, Hkv, false) ||
        !valid_heads(out, a, Tq, Hq, true) || !d_q_offsets || !d_k_offsets || !valid_scale(scale))
        return PICASSO_ERR_INVALID_ARG;
    const ForwardPlan p = forward_plan(a);
    const size_t need = attention_forward_bytes(a, p);
    const size_t offsets = ((size_t)B + 1) * 4;
    if (!apart({span(q, a, Tq, Hq, false), span(k, a, Tk, Hkv, false), span(v, a, Tk, Hkv, false), whole(d_q_offsets, offsets, false),
                whole(d_k_offsets, offsets, false), span(out, a, Tq, Hq, true), whole(d_lse, (size_t)Tq * Hq * 4, true),
                whole(d_workspace, std::min(need, workspace_bytes), true)}))
        return PICASSO_ERR_INVALID_ARG;
    if (need && (!d_workspace || workspace_bytes < need || !aligned(d_workspace, 16))) return PICASSO_ERR_WORKSPACE;
    if (Tq == 0) return PICASSO_OK;
    hipStream_t s = (hipStream_t)stream;
    ON_DEVICE(c);
    const attn::Offsets off{d_q_offsets, d_k_offsets, B, Tq, Tk};
    const attn::Group group = attn::heads_per_group(a.G());
    float* part_out = p.splits > 1 ? (float*)d_workspace : nullptr;
    float* part_lse = p.splits > 1 ? (float*)((char*)d_workspace + up((size_t)p.splits * Tq * Hq * D * 4)) : nullptr;
    const float scale2 = scale * attn::LOG2E;
#define PICASSO_FORWARD(T, DP, W)                                                                                          \
    attn::forward_kernel<T, DP, W>                                                                                         \
        <<<dim3((unsigned)attn::tile_numbers(Tq, a.G(), 32 * W, B), Hkv, p.splits), feat::BLOCK, 0, s>>>(                   \
            heads<const T>(q), heads<const T>(k), heads<const T>(v), off, Hq, Hkv, group, D, causal, clear_outside, scale2, \
            heads<T>(out), d_lse, part_out, part_lse)
#define PICASSO_WIDTH(T, DP)                               \
    if (p.row_waves == 4) PICASSO_FORWARD(T, DP, 4);       \
    else PICASSO_FORWARD(T, DP, 1)
#define PICASSO_CALL(T)                                                                                                       \
    FOR_WIDTH(T, D, PICASSO_WIDTH);                                                                                           \
    if (p.splits > 1)                                                                                                         \
    attn::join_kernel<T><<<groups_for((long long)Tq * Hq * (D / 4)), feat::BLOCK, 0, s>>>(                                      \
        part_out, part_lse, p.splits, off, Hq, D, clear_outside, heads<T>(out), d_lse)
    FOR_TYPE(type, PICASSO_CALL);
#undef PICASSO_CALL
#undef PICASSO_WIDTH
#undef PICASSO_FORWARD
    LAUNCHED(c);
    return PICASSO_OK;
}

int picasso_attention_backward(picasso_ctx* c, void* stream, int type, const picasso_heads* gout, const picasso_heads* q,
                               const picasso_heads* k, const picasso_heads* v, const picasso_heads* out, const float* d_lse,
                               const int32_t* d_q_offsets, const int32_t* d_k_offsets, int32_t B, int32_t Tq, int32_t Tk, int32_t Hq,
                               int32_t Hkv, int32_t D, int causal, float scale, int clear_outside, const picasso_heads* gq,
                               const picasso_heads* gk, const picasso_heads* gv, void* d_workspace, size_t workspace_bytes) {
    const Attention a{type, B, Tq, Tk, Hq, Hkv, D};
    if (!c || !valid(a) || !valid_heads(gout, a, Tq, Hq, false) || !valid_heads(q, a, Tq, Hq, false) || !valid_heads(k, a, Tk, Hkv, false) ||
        !valid_heads(v, a, Tk, Hkv, false) || !valid_heads(out, a, Tq, Hq, false) || !valid_heads(gq, a, Tq, Hq, true) ||
        !valid_heads(gk, a, Tk, Hkv, true) || !valid_heads(gv, a, Tk, Hkv, true) || (Tq > 0 && !d_lse) || !d_q_offsets || !d_k_offsets || !valid_scale(scale))
        return PICASSO_ERR_INVALID_ARG;
    const BackwardPlan p = backward_plan(a);
    const size_t need = attention_backward_bytes(a, p), offsets = ((size_t)B + 1) * 4;
    if (!apart({span(gout, a, Tq, Hq, false), span(q, a, Tq, Hq, false), span(k, a, Tk, Hkv, false), span(v, a, Tk, Hkv, false),
                span(out, a, Tq, Hq, false), whole(d_lse, (size_t)Tq * Hq * 4, false), whole(d_q_offsets, offsets, false),
                whole(d_k_offsets, offsets, false), span(gq, a, Tq, Hq, true), span(gk, a, Tk, Hkv, true), span(gv, a, Tk, Hkv, true),
                whole(d_workspace, std::min(need, workspace_bytes), true)}))
        return PICASSO_ERR_INVALID_ARG;
    if (!d_workspace || workspace_bytes < need || !aligned(d_workspace, 16)) return PICASSO_ERR_WORKSPACE;
    if (Tq == 0 && Tk == 0) return PICASSO_OK;
    hipStream_t s = (hipStream_t)stream;
    ON_DEVICE(c);
    const attn::Offsets off{d_q_offsets, d_k_offsets, B, Tq, Tk};
    const attn::Group group = attn::heads_per_group(a.G());
    const attn::Scale sc{scale * attn::LOG2E, scale};
    float* delta = (float*)d_workspace;
    float* part = (float*)((char*)d_workspace + up((size_t)Tq * Hq * 4));
    float* part_v = p.key_splits > 1 ? (float*)((char*)part + up((size_t)p.key_splits * Tk * Hkv * D * 4)) : nullptr;
#define PICASSO_KEYS(T, DP)                                                                                                       \
    attn::backward_keys_kernel<T, DP><<<dim3((unsigned)attn::tile_numbers(Tk, 1, 128, B), Hkv, p.key_splits), feat::BLOCK, 0, s>>>( \
        heads<const T>(gout), heads<const T>(q), heads<const T>(k), heads<const T>(v), d_lse, delta, off, Hq, Hkv, group, D,        \
        causal, clear_outside, sc, heads<T>(gk), heads<T>(gv), part, part_v)
#define PICASSO_QUERIES(T, DP)                                                                                                      \
    attn::backward_queries_kernel<T, DP>                                                                                            \
        <<<dim3((unsigned)attn::tile_numbers(Tq, a.G(), 128, B), Hkv, p.query_splits), feat::BLOCK, 0, s>>>(                        \
            heads<const T>(gout), heads<const T>(q), heads<const T>(k), heads<const T>(v), d_lse, delta, off, Hq, Hkv, group, D,      \
            causal, clear_outside, sc, heads<T>(gq), part)
#define PICASSO_SUM(T, splits, part, offsets, rows, H, to)                                                                         \
    attn::sum_kernel<T><<<groups_for((long long)(rows) * (H) * (D / 4)), feat::BLOCK, 0, s>>>(                                        \
        part, splits, offsets, B, rows, H, D, clear_outside, heads<T>(to))
#define PICASSO_CALL(T)                                                                    \
    attn::delta_kernel<T><<<groups_for((long long)Tq * Hq * 16), feat::BLOCK, 0, s>>>(heads<const T>(gout), heads<const T>(out), Tq, Hq, D, delta)
    if (Tq > 0) {
        FOR_TYPE(type, PICASSO_CALL);
        LAUNCHED(c);  // (what follows reads it)
    }
#undef PICASSO_CALL
#define PICASSO_CALL(T)                                                                                              \
    if (Tk > 0) {                                                                                                    \
        FOR_WIDTH(T, D, PICASSO_KEYS);                                                                               \
        if (p.key_splits > 1) {                                                                                      \
            PICASSO_SUM(T, p.key_splits, part, d_k_offsets, Tk, Hkv, gk);                                            \
            PICASSO_SUM(T, p.key_splits, part_v, d_k_offsets, Tk, Hkv, gv);                                          \
        }                                                                                                            \
    }                                                                                                                \
    if (Tq > 0) {                                                                                                    \
        FOR_WIDTH(T, D, PICASSO_QUERIES);                                                                            \
        if (p.query_splits > 1) PICASSO_SUM(T, p.query_splits, part, d_q_offsets, Tq, Hq, gq);                       \
    }
    FOR_TYPE(type, PICASSO_CALL);
#undef PICASSO_CALL
#undef PICASSO_SUM
#undef PICASSO_QUERIES
#undef PICASSO_KEYS
    LAUNCHED(c);
    return PICASSO_OK;
}

size_t picasso_gradients_workspace_bytes(int32_t n, const int64_t* h_sizes) {
    if (n < 0 || (n > 0 && !h_sizes) || !countable(n, h_sizes)) return 0;
    size_t partials = 0;
    gradient_tables(n, nullptr, nullptr, h_sizes, nullptr, [&](const grads::Table&, int groups) { partials += groups; });
    // (and their sum, where it is made first)
    return std::max<size_t>(partials + (partials > grads::MAX_PARTIALS), 1) * sizeof(double);
}

int picasso_gradient_norm(picasso_ctx* c, void* stream, int32_t n, const void* const* h_grads, const int64_t* h_sizes,
                          const int32_t* h_types, float* d_norm, void* d_workspace, size_t workspace_bytes) {
    if (!c || !valid_gradients(n, h_grads, h_sizes, h_types) || !d_norm) return PICASSO_ERR_INVALID_ARG;
    const size_t need = picasso_gradients_workspace_bytes(n, h_sizes);
    if (const int rc = tensors_apart(n, h_grads, nullptr, h_sizes, h_types, d_norm, d_workspace, std::min(need, workspace_bytes))) return rc;
    if (!d_workspace || !aligned(d_workspace, 8) || workspace_bytes < need) return PICASSO_ERR_WORKSPACE;
    hipStream_t s = (hipStream_t)stream;
    ON_DEVICE(c);
    double* ws = (double*)d_workspace;
    const int partials = queue_squares(s, n, h_grads, h_sizes, h_types, ws);
    grads::norm_kernel<<<1, feat::BLOCK, 0, s>>>(ws, partials, d_norm);
    LAUNCHED(c);
    return PICASSO_OK;
}

int picasso_clip_gradients(picasso_ctx* c, void* stream, int32_t n, const void* const* h_grads, const int64_t* h_sizes,
                           const int32_t* h_types, double max_norm, void* const* h_out, float* d_norm, void* d_workspace,
                           size_t workspace_bytes) {
    if (!c || !valid_gradients(n, h_grads, h_sizes, h_types) || !(max_norm >= 0.0) || (n > 0 && !h_out)) return PICASSO_ERR_INVALID_ARG;
    for (int k = 0; k < n; ++k)
        if ((h_sizes[k] > 0 && !h_out[k]) || !aligned(h_out[k], size_of(h_types[k]))) return PICASSO_ERR_INVALID_ARG;
    const size_t need = picasso_gradients_workspace_bytes(n, h_sizes);
    if (const int rc = tensors_apart(n, h_grads, h_out, h_sizes, h_types, d_norm, d_workspace, std::min(need, workspace_bytes))) return rc;
    if (!d_workspace || !aligned(d_workspace, 8) || workspace_bytes < need) return PICASSO_ERR_WORKSPACE;
    hipStream_t s = (hipStream_t)stream;
    ON_DEVICE(c);
    double* ws = (double*)d_workspace;
    int partials = queue_squares(s, n, h_grads, h_sizes, h_types, ws);
    if (partials > grads::MAX_PARTIALS) {
        grads::total_kernel<<<1, feat::BLOCK, 0, s>>>(ws, partials, ws + partials);
        ws += partials;
        partials = 1;
    }
    bool first = true;
    gradient_tables(n, h_grads, h_out, h_sizes, h_types, [&](const grads::Table& t, int groups) {
        grads::scale_kernel<<<groups, feat::BLOCK, 0, s>>>(t, ws, partials, max_norm, first ? d_norm : nullptr);
        first = false;
    });
    if (first && d_norm) grads::norm_kernel<<<1, feat::BLOCK, 0, s>>>(ws, 0, d_norm);  // (nothing to scale)
    LAUNCHED(c);
    return PICASSO_OK;
}

}  // extern "C"
