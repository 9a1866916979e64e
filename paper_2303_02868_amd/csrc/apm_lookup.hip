// Rows of a table for each token, y[t] = scale sum w[p] table[ids[p]], and the gradients of that.  HBM-bound, all of it.
//
// Forward, a lane has eight columns of a token and adds up its rows.  The gradient of the table goes by the sorted positions, so that each of its rows is
// written once and nothing is added atomically: the sorted positions are cut into chunks of equal size, whatever rows they belong to, a wavefront adds up what it
// has of each row, and a row that goes beyond a chunk is put together from the chunks' parts, in their order.
#include <algorithm>

#include "apm_tok.h"

namespace apm {
namespace {

constexpr int kWave = 64, kThreads = 256, kWaves = kThreads / kWave;

struct LookupArgs {
    const void* ids;
    const char* table;
    char* y;
    apm_vector weights;
    int64_t table_stride, y_stride;
    int64_t first_token;  // of the launch
    uint32_t tokens, vecs;
    float inv_vecs;
    int32_t cols;
    uint32_t rows;
    int32_t per_token, id_type, accumulate;
    float scale;
};

__device__ __forceinline__ float weight_of(const apm_vector& w, int64_t p) { return w.data ? load1(w.data, w.dtype, p) : 1.0f; }

constexpr int kRowsAhead = 4;  // of a token's rows, loads under way
template <class T, class Y, int UNROLL>
__global__ __launch_bounds__(kThreads) void apm_lookup_kernel(LookupArgs a) {
    const uint32_t first = blockIdx.x * (uint32_t)(kThreads * UNROLL), row0 = first / a.vecs, vec0 = first - row0 * a.vecs;
    auto place = [&](int u) { return VecPlace(row0, vec0, (uint32_t)(u * kThreads) + threadIdx.x, a.vecs, a.inv_vecs, a.cols); };
    float sum[UNROLL][kVec];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u)
#pragma unroll
        for (int i = 0; i < kVec; ++i) sum[u][i] = 0.0f;
    constexpr int AHEAD = UNROLL > 1 ? 1 : kRowsAhead;
    for (int j = 0; j < a.per_token; j += AHEAD) {
        Raw<T> x[UNROLL][AHEAD];
        float w[UNROLL][AHEAD];
        bool there[UNROLL][AHEAD];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const VecPlace at = place(u);
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const int64_t p = (a.first_token + at.row) * a.per_token + j + k;
                const bool in = at.row < a.tokens && j + k < a.per_token;
                const uint32_t row = in ? row_of(a.ids, a.id_type, p, a.rows) : a.rows;
                there[u][k] = row < a.rows;
                w[u][k] = there[u][k] ? weight_of(a.weights, p) : 0.0f;
                x[u][k].load(a.table + (int64_t)row * a.table_stride * (int64_t)sizeof(T), at.col, there[u][k] ? at.n : 0);
            }
        }
#pragma unroll
        for (int u = 0; u < UNROLL; ++u)
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
                if (there[u][k]) {
#pragma unroll
                    for (int i = 0; i < kVec; ++i) sum[u][i] = fmaf(w[u][k], x[u][k][i], sum[u][i]);
                }
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
        const VecPlace at = place(u);
        char* y = a.y + (a.first_token + at.row) * a.y_stride * (int64_t)sizeof(Y);
        const int n = at.row < a.tokens ? at.n : 0;
        float v[kVec];
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = sum[u][i] * a.scale;
        if (a.accumulate) {
            Raw<Y> old;
            old.load(y, at.col, n);
#pragma unroll
            for (int i = 0; i < kVec; ++i) v[i] += old[i];
        }
        store8<Y>(y, at.col, n, v);
    }
}

int check_lookup(const apm_lookup& l, bool forward) {
    if (l.tokens < 0 || l.tokens > APM_MAX_POSITIONS || l.per_token < 1 || l.per_token > APM_MAX_POSITIONS || l.tokens * l.per_token > APM_MAX_POSITIONS || l.rows < 1 ||
        l.rows > APM_MAX_POSITIONS || l.cols < 1 || l.cols > kMostCols)
        return fail(APM_EINVAL, "bad size: %lld tokens, %lld rows of a token, table of %lld x %lld", (long long)l.tokens, (long long)l.per_token, (long long)l.rows, (long long)l.cols);
    if (l.tokens == 0) return APM_OK;
    int rc = check_indices("ids", l.ids);
    if (rc == APM_OK) rc = check_vector("weights", l.weights);
    if (rc == APM_OK && forward) rc = check_matrix("table", l.table, l.rows, l.cols, false);
    if (rc == APM_OK && forward) rc = check_matrix("y", l.y, l.tokens, l.cols, true);
    return rc;
}

int forward(const apm_lookup* lp, void* stream) {
    if (!lp) return fail(APM_EINVAL, "missing argument");
    const apm_lookup& l = *lp;
    const int rc = check_lookup(l, true);
    if (rc != APM_OK || l.tokens == 0) return rc;
    LookupArgs a{};
    a.ids = l.ids.data, a.id_type = l.ids.type, a.table = (const char*)l.table.data, a.y = (char*)l.y.data, a.weights = l.weights;
    a.table_stride = l.table.stride, a.y_stride = l.y.stride;
    a.vecs = (uint32_t)div_up(l.cols, kVec), a.inv_vecs = 1.0f / (float)a.vecs, a.cols = (int32_t)l.cols;
    a.rows = (uint32_t)l.rows, a.per_token = (int32_t)l.per_token, a.accumulate = l.accumulate, a.scale = (float)l.scale;
    const int64_t most = std::max<int64_t>(1, kMostVecs / a.vecs);
    for (a.first_token = 0; a.first_token < l.tokens; a.first_token += most) {
        a.tokens = (uint32_t)std::min(most, l.tokens - a.first_token);
        const hipStream_t s = (hipStream_t)stream;
        auto start = [&](auto kernel, int unroll) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)div_up((int64_t)a.tokens * a.vecs, kThreads * unroll)), dim3(kThreads), 0, s, a);
        };
        auto with = [&](auto t, auto y) {
            typedef decltype(t) T;
            typedef decltype(y) Y;
            if (a.per_token == 1) start(apm_lookup_kernel<T, Y, 2>, 2);
            else start(apm_lookup_kernel<T, Y, 1>, 1);
        };
        if (l.table.dtype == APM_F32) l.y.dtype == APM_F32 ? with(float(), float()) : with(float(), bf16());
        else l.y.dtype == APM_F32 ? with(bf16(), float()) : with(bf16(), bf16());
        APM_HIP(hipGetLastError());
    }
    return APM_OK;
}

// ---- the gradient of the table ------------------------------------------------------------------
constexpr int kChunk = 64;                  // sorted positions of a wavefront, one of each lane to begin with
constexpr int kSlice = kWave * kVec;        // columns of a wavefront
constexpr int kAhead = 8;                   // rows of dy under way
constexpr int kEmptyRows = 32;              // rows of dtable that a wavefront looks through for those without positions

struct TableGradArgs {
    const void* ids;
    const char* dy;
    char* dtable;
    const int32_t* order;
    const int64_t* offsets;
    float* parts;  // [chunks][2][cols_8]: of the row that began before the chunk, and of the row that goes on behind it
    apm_vector weights;
    int64_t dy_stride, table_stride;
    uint32_t n, rows, per_token, chunks, slices, empty;  // empty: wavefronts that write zeros
    uint32_t first_item;
    int32_t cols, cols_8, id_type, accumulate;
    float scale;
};

template <class T, bool NT = true> __device__ __forceinline__ void finish_row(const TableGradArgs& a, uint32_t row, int col, int n, float (&v)[kVec]) {
    char* to = a.dtable + (int64_t)row * a.table_stride * (int64_t)sizeof(T);
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] *= a.scale;
    if (a.accumulate) {
        Raw<T> old;
        old.load(to, col, n);
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] += old[i];
    }
    store8<T, NT>(to, col, n, v);
}
__device__ __forceinline__ float* part_of(const TableGradArgs& a, uint32_t chunk, int which, int col) {
    return a.parts + ((uint64_t)chunk * 2 + (uint32_t)which) * (uint32_t)a.cols_8 + (uint32_t)col;
}
__device__ __forceinline__ uint32_t row_at(const TableGradArgs& a, uint32_t i) {
    const uint32_t p = (uint32_t)a.order[i];
    return p < a.n ? row_of(a.ids, a.id_type, p, a.rows) : a.rows;
}

template <class D, class T>
__global__ __launch_bounds__(kThreads) void apm_table_grad_kernel(TableGradArgs a) {
    const int lane = (int)threadIdx.x % kWave;
    const uint32_t item = a.first_item + (uint32_t)__builtin_amdgcn_readfirstlane((int)(blockIdx.x * kWaves + threadIdx.x / kWave));
    const uint32_t summing = a.chunks * a.slices;
    if (item >= summing) {  // rows without positions
        const uint32_t e = item - summing;
        if (e >= a.empty) return;
        const uint32_t first = e * kEmptyRows, r = first + (uint32_t)lane;
        const bool none = lane < kEmptyRows && r < a.rows && a.offsets[r] >= a.offsets[r + 1];
        uint64_t mask = __ballot(none);
        const float zero[kVec] = {};
        while (mask) {
            const uint32_t row = first + (uint32_t)__builtin_ctzll(mask);
            mask &= mask - 1;
            for (int col = lane * kVec; col < a.cols; col += kSlice) store8<T, true>(a.dtable + (int64_t)row * a.table_stride * (int64_t)sizeof(T), col, min(kVec, a.cols - col), zero);
        }
        return;
    }
    const uint32_t chunk = item / a.slices, start = chunk * kChunk;
    const int col = (int)(item - chunk * a.slices) * kSlice + lane * kVec, there = max(0, min(kVec, a.cols - col)), n = (int)min((uint32_t)kChunk, a.n - start);
    // lane l: the chunk's l-th position
    uint32_t my_row = a.rows, my_token = 0;
    float my_weight = 0.0f;
    if (lane < n) {
        const uint32_t p = (uint32_t)a.order[start + (uint32_t)lane];
        if (p < a.n) {
            my_row = row_of(a.ids, a.id_type, p, a.rows);
            my_token = p / a.per_token;
            if (my_row < a.rows) my_weight = weight_of(a.weights, p);
        }
    }
    auto of_lane = [](uint32_t v, int l) { return (uint32_t)__builtin_amdgcn_readlane((int)v, l); };
    uint32_t row = of_lane(my_row, 0);
    if (row >= a.rows) return;  // so are all behind it
    bool before = start > 0 && row_at(a, start - 1) == row;  // the row began in an earlier chunk
    const uint32_t after = start + kChunk < a.n ? row_at(a, start + kChunk) : a.rows;
    float sum[kVec] = {};
    auto flush = [&](bool goes_on) {
        if (!before && !goes_on) return finish_row<T>(a, row, col, there, sum);
        if (there <= 0) return;
        u32x4 w[2];
#pragma unroll
        for (int i = 0; i < kVec; ++i) w[i / 4][i % 4] = __builtin_bit_cast(uint32_t, sum[i]);
        u32x4* to = (u32x4*)part_of(a, chunk, before ? 0 : 1, col);
        to[0] = w[0], to[1] = w[1];
    };
    for (int i0 = 0; i0 < n; i0 += kAhead) {
        Raw<D> x[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int i = i0 + k;
            const bool in = i < n && of_lane(my_row, i & (kWave - 1)) < a.rows;
            x[k].load(a.dy + (int64_t)of_lane(my_token, i & (kWave - 1)) * a.dy_stride * (int64_t)sizeof(D), col, in ? there : 0);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int i = i0 + k;
            if (i >= n) break;
            const uint32_t r = of_lane(my_row, i);
            if (r != row) {
                flush(false);
                if (r >= a.rows) return;
                row = r, before = false;
#pragma unroll
                for (int e = 0; e < kVec; ++e) sum[e] = 0.0f;
            }
            const float w = __builtin_bit_cast(float, of_lane(__builtin_bit_cast(uint32_t, my_weight), i));
#pragma unroll
            for (int e = 0; e < kVec; ++e) sum[e] = fmaf(w, x[k][e], sum[e]);
        }
    }
    flush(after == row);
}

// A row that goes beyond the chunk in which it begins: that chunk's part and those of the chunks behind it.
template <class T>
__global__ __launch_bounds__(kThreads) void apm_table_grad_join_kernel(TableGradArgs a) {
    const int lane = (int)threadIdx.x % kWave;
    const uint32_t item = a.first_item + (uint32_t)__builtin_amdgcn_readfirstlane((int)(blockIdx.x * kWaves + threadIdx.x / kWave));
    if (item >= a.chunks * a.slices) return;
    const uint32_t chunk = item / a.slices, start = chunk * kChunk, next = start + kChunk;
    if (next >= a.n) return;
    const uint32_t row = row_at(a, next - 1);
    if (row >= a.rows || row_at(a, next) != row) return;
    if (start > 0 && row_at(a, start - 1) == row) return;  // began earlier still
    const int64_t end = min(max(a.offsets[row + 1], (int64_t)next + 1), (int64_t)a.n);
    const uint32_t last = (uint32_t)(end - 1) / kChunk;
    const int col = (int)(item - chunk * a.slices) * kSlice + lane * kVec, there = max(0, min(kVec, a.cols - col));
    if (there <= 0) return;
    float sum[kVec];
    {
        const float* p = part_of(a, chunk, 1, col);
#pragma unroll
        for (int i = 0; i < kVec; ++i) sum[i] = p[i];
    }
    for (uint32_t c = chunk + 1; c <= last; c += 4) {
        Raw<float> x[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k].load(part_of(a, min(c + (uint32_t)k, last), 0, 0), col, c + (uint32_t)k <= last ? kVec : 0);
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int i = 0; i < kVec; ++i) sum[i] += x[k][i];
    }
    finish_row<T>(a, row, col, there, sum);
}

// ---- the gradient of the weights ----------------------------------------------------------------
struct WeightGradArgs {
    const void* ids;
    const char* dy;
    const char* table;
    apm_vector dweights;
    int64_t dy_stride, table_stride;
    int64_t n, first;
    int32_t per_token, cols, id_type;
    uint32_t rows;
    float scale;
};
template <class D, class T>
__global__ __launch_bounds__(kThreads) void apm_lookup_weights_kernel(WeightGradArgs a) {
    const int lane = (int)threadIdx.x % kWave;
    const int64_t p = a.first + (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    if (p >= a.n) return;
    const uint32_t row = row_of(a.ids, a.id_type, p, a.rows);
    float sum = 0.0f;
    if (row < a.rows) {
        const char* dy = a.dy + p / a.per_token * a.dy_stride * (int64_t)sizeof(D);
        const char* x = a.table + (int64_t)row * a.table_stride * (int64_t)sizeof(T);
#pragma unroll 2
        for (int col = lane * kVec; col < a.cols; col += kSlice) {
            const int n = min(kVec, a.cols - col);
            Raw<D> d;
            Raw<T> t;
            d.load(dy, col, n);
            t.load(x, col, n);
#pragma unroll
            for (int i = 0; i < kVec; ++i) sum = fmaf(d[i], t[i], sum);
        }
        sum = wave_sum(sum) * a.scale;
    }
    if (lane == 0) store1(a.dweights.data, a.dweights.dtype, p, sum);
}

size_t room_of(const apm_lookup& l) {
    return (size_t)div_up(l.tokens * l.per_token, kChunk) * 2 * (size_t)div_up(l.cols, kVec) * kVec * sizeof(float);
}

int backward(const apm_lookup* lp, const apm_lookup_grads* gp, void* workspace, size_t workspace_bytes, void* stream) {
    if (!lp || !gp) return fail(APM_EINVAL, "missing argument");
    const apm_lookup& l = *lp;
    const apm_lookup_grads& g = *gp;
    const int64_t n = l.tokens * l.per_token;
    int rc = check_lookup(l, false);
    if (rc == APM_OK) rc = check_matrix("dy", g.dy, l.tokens, l.cols, false);
    if (rc == APM_OK && g.dtable.data) {
        rc = check_matrix("dtable", g.dtable, l.rows, l.cols, true);
        if (rc == APM_OK && (!g.offsets || (!g.order && n > 0))) rc = fail(APM_EINVAL, "dtable needs order and offsets");
        if (rc == APM_OK && (!aligned_to(g.order, 4) || !aligned_to(g.offsets, 8))) rc = fail(APM_EINVAL, "order or offsets are not aligned to their elements");
        if (rc == APM_OK) rc = check_room(workspace, workspace_bytes, room_of(l));
    }
    if (rc == APM_OK && g.dweights.data) {
        rc = check_vector("dweights", g.dweights);
        if (rc == APM_OK && n > 0) rc = check_matrix("table", l.table, l.rows, l.cols, false);
    }
    if (rc != APM_OK) return rc;
    const hipStream_t s = (hipStream_t)stream;
    const int64_t most_items = max_workgroups(kThreads) * kWaves / 2;
    if (g.dtable.data) {
        TableGradArgs a{};
        a.ids = l.ids.data, a.id_type = l.ids.type, a.dy = (const char*)g.dy.data, a.dtable = (char*)g.dtable.data, a.order = g.order, a.offsets = g.offsets;
        a.parts = (float*)workspace, a.weights = l.weights, a.dy_stride = g.dy.stride, a.table_stride = g.dtable.stride;
        a.n = (uint32_t)n, a.rows = (uint32_t)l.rows, a.per_token = (uint32_t)l.per_token, a.cols = (int32_t)l.cols, a.cols_8 = (int32_t)(div_up(l.cols, kVec) * kVec);
        a.chunks = (uint32_t)div_up(n, kChunk), a.slices = (uint32_t)div_up(l.cols, kSlice), a.empty = g.accumulate ? 0 : (uint32_t)div_up(l.rows, kEmptyRows);
        a.accumulate = g.accumulate, a.scale = (float)l.scale;
        const int64_t summing = (int64_t)a.chunks * a.slices, items = summing + a.empty;
        if (items > INT32_MAX) return fail(APM_EINVAL, "too many positions for so many columns");
        for (int64_t at = 0; at < items; at += most_items) {
            a.first_item = (uint32_t)at;
            const dim3 grid((unsigned)div_up(std::min(most_items, items - at), kWaves)), block(kThreads);
            auto start = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, s, a); };
            const bool wide = g.dtable.dtype == APM_F32;
            if (n > 0 && g.dy.dtype == APM_F32) wide ? start(apm_table_grad_kernel<float, float>) : start(apm_table_grad_kernel<float, bf16>);
            else wide ? start(apm_table_grad_kernel<bf16, float>) : start(apm_table_grad_kernel<bf16, bf16>);
            APM_HIP(hipGetLastError());
        }
        if (a.chunks > 1) {
            for (int64_t at = 0; at < summing; at += most_items) {
                a.first_item = (uint32_t)at;
                const dim3 grid((unsigned)div_up(std::min(most_items, summing - at), kWaves)), block(kThreads);
                if (g.dtable.dtype == APM_F32) hipLaunchKernelGGL(apm_table_grad_join_kernel<float>, grid, block, 0, s, a);
                else hipLaunchKernelGGL(apm_table_grad_join_kernel<bf16>, grid, block, 0, s, a);
                APM_HIP(hipGetLastError());
            }
        }
    }
    if (g.dweights.data && n > 0) {
        WeightGradArgs a{};
        a.ids = l.ids.data, a.id_type = l.ids.type, a.dy = (const char*)g.dy.data, a.table = (const char*)l.table.data, a.dweights = g.dweights;
        a.dy_stride = g.dy.stride, a.table_stride = l.table.stride, a.n = n, a.per_token = (int32_t)l.per_token, a.cols = (int32_t)l.cols;
        a.rows = (uint32_t)l.rows, a.scale = (float)l.scale;
        for (a.first = 0; a.first < n; a.first += most_items) {
            const dim3 grid((unsigned)div_up(std::min(most_items, n - a.first), kWaves)), block(kThreads);
            auto start = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, s, a); };
            const bool wide = l.table.dtype == APM_F32;
            if (g.dy.dtype == APM_F32) wide ? start(apm_lookup_weights_kernel<float, float>) : start(apm_lookup_weights_kernel<float, bf16>);
            else wide ? start(apm_lookup_weights_kernel<bf16, float>) : start(apm_lookup_weights_kernel<bf16, bf16>);
            APM_HIP(hipGetLastError());
        }
    }
    return APM_OK;
}

}  // namespace
}  // namespace apm

extern "C" int apm_lookup_forward(const apm_lookup* l, void* stream) {
    return apm::guarded([&]() -> int { return apm::forward(l, stream); });
}

extern "C" size_t apm_lookup_workspace_bytes(const apm_lookup* l) { return !l || apm::check_lookup(*l, false) != APM_OK ? 0 : apm::room_of(*l); }

extern "C" int apm_lookup_backward(const apm_lookup* l, const apm_lookup_grads* g, void* workspace, size_t workspace_bytes, void* stream) {
    return apm::guarded([&]() -> int { return apm::backward(l, g, workspace, workspace_bytes, stream); });
}
