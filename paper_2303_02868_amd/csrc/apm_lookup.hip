// Rows of a table for each token, y[t] = scale sum w[p] table[ids[p]], and the gradients of that.  HBM-bound, all of it.
//
// Forward, a wavefront has 512 columns of a few tokens and adds up their rows.  The gradient of the table goes by the sorted positions, so that each of its rows is
// written once and nothing is added atomically: the sorted positions are cut into chunks of equal size, whatever rows they belong to, a wavefront adds up what it
// has of each row, and a row that goes beyond a chunk is put together from the chunks' parts, in their order.
#include <algorithm>
#include <type_traits>

#include "apm_tok.h"

namespace apm {
namespace {

constexpr int kWave = 64, kThreads = 256, kWaves = kThreads / kWave;

constexpr int kSlice = kWave * kVec;                        // columns of a wavefront
constexpr int kTokens = 4, kTurn = kWave / kTokens;         // tokens of a wavefront, whose loads are under way together; ids of a token that it takes at a time

struct LookupArgs {
    const void* ids;
    apm_matrix table, y;
    apm_vector weights;
    int64_t first, end;  // tokens of this launch
    uint32_t slices, rows;
    int32_t cols, per_token, id_type, accumulate;
    float scale;
};

__device__ __forceinline__ float weight_of(const apm_vector& w, int64_t p) { return w.data ? load1(w.data, w.dtype, p) : 1.0f; }
__device__ __forceinline__ uint32_t of_lane(uint32_t v, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)v, lane); }
__device__ __forceinline__ float of_lane(float v, int lane) { return __builtin_bit_cast(float, of_lane(__builtin_bit_cast(uint32_t, v), lane)); }

// 16384 tokens of a 50257 x 2048 table: 18.0 us = 5.2 TB/s of what has to move; back from experts, 8191 tokens of two weighted rows of 1024, to fp32: 11.7 = 5.7.  Stores
// are non-temporal, so that the rows that come often stay in L2 (22.8 us without), loads are not (24.8 with); two tokens a wavefront 17.7 and 12.0, eight 18.2 and 11.5.
template <class T, class Y>
__global__ __launch_bounds__(kThreads) void apm_lookup_kernel(LookupArgs a) {
    const int lane = (int)threadIdx.x % kWave;
    const uint32_t item = blockIdx.x * kWaves + (uint32_t)__builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), nth = item / a.slices;
    const int64_t t0 = a.first + (int64_t)nth * kTokens;
    if (t0 >= a.end) return;
    LaneCols l;
    l.set((int)(item - nth * a.slices) * kSlice + lane * kVec, a.cols);
    float sum[kTokens][kVec] = {};
    for (int j0 = 0; j0 < a.per_token; j0 += kTurn) {
        const int64_t t = t0 + lane / kTurn, j = j0 + lane % kTurn;
        uint32_t my_row = a.rows;
        float my_weight = 0.0f;
        if (t < a.end && j < a.per_token) {
            const int64_t p = t * a.per_token + j;
            my_row = row_of(a.ids, a.id_type, p, a.rows);
            if (my_row < a.rows) my_weight = weight_of(a.weights, p);
        }
        const int turn = min(kTurn, a.per_token - j0);
        for (int k = 0; k < turn; ++k) {
            Raw<T> x[kTokens];
#pragma unroll
            for (int u = 0; u < kTokens; ++u) {  // no such row: zeros, by a factor of zero
                const uint32_t row = of_lane(my_row, u * kTurn + k);
                load_row<0>(x[u], a.table, row, a.cols, row < a.rows, l);
            }
#pragma unroll
            for (int u = 0; u < kTokens; ++u) {
                const float w = of_lane(my_weight, u * kTurn + k);
                settle(x[u], l, a.cols);
#pragma unroll
                for (int i = 0; i < kVec; ++i) sum[u][i] = fmaf(w, x[u][i], sum[u][i]);
            }
        }
    }
#pragma unroll
    for (int u = 0; u < kTokens; ++u) {
        const bool there = t0 + u < a.end;
        float v[kVec];
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = sum[u][i] * a.scale;
        if (a.accumulate) {
            Raw<Y> old;
            load_row(old, a.y, t0 + u, a.cols, there, l);
            settle(old, l, a.cols);
#pragma unroll
            for (int i = 0; i < kVec; ++i) v[i] += old[i];
        }
        store_row<Y>(a.y, t0 + u, a.cols, there, l, v);
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
    a.ids = l.ids.data, a.id_type = l.ids.type, a.table = l.table, a.y = l.y, a.weights = l.weights;
    a.slices = (uint32_t)div_up(l.cols, kSlice), a.cols = (int32_t)l.cols;
    a.rows = (uint32_t)l.rows, a.per_token = (int32_t)l.per_token, a.accumulate = l.accumulate, a.scale = (float)l.scale;
    const int64_t most = std::max<int64_t>(1, workgroups_of_launch(kThreads) * kWaves / a.slices) * kTokens;  // tokens of a launch
    for (a.first = 0; a.first < l.tokens; a.first = a.end) {
        a.end = std::min(l.tokens, a.first + most);  // the last workgroup can have wavefronts to spare, whose tokens are the next launch's: with accumulate they would be added twice
        const dim3 grid((unsigned)div_up(div_up(a.end - a.first, kTokens) * a.slices, kWaves)), block(kThreads);
        const hipStream_t s = (hipStream_t)stream;
        auto start = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, s, a); };
        if (l.table.dtype == APM_F32) l.y.dtype == APM_F32 ? start(apm_lookup_kernel<float, float>) : start(apm_lookup_kernel<float, bf16>);
        else l.y.dtype == APM_F32 ? start(apm_lookup_kernel<bf16, float>) : start(apm_lookup_kernel<bf16, bf16>);
        APM_HIP(hipGetLastError());
    }
    return APM_OK;
}

// ---- the gradient of the weights ----------------------------------------------------------------
struct WeightGradArgs {
    const void* ids;
    apm_matrix dy, table;
    apm_vector dweights;
    uint32_t n, per_token, rows;
    int32_t cols, id_type;
    float scale;
};
// Of one position, by a wavefront.
template <class D, class T> __device__ __forceinline__ void weight_grad(const WeightGradArgs& a, uint32_t p, int lane) {
    const uint32_t row = (uint32_t)__builtin_amdgcn_readfirstlane((int)row_of(a.ids, a.id_type, p, a.rows));
    float sum = 0.0f;
    if (row < a.rows) {
        const uint32_t token = p / a.per_token;
        constexpr int kSlices = 2;  // under way
        for (int col = 0; col < a.cols; col += kSlices * kSlice) {
            LaneCols l[kSlices];
            Raw<D> d[kSlices];
            Raw<T> t[kSlices];
#pragma unroll
            for (int s = 0; s < kSlices; ++s) {
                l[s].set(col + s * kSlice + lane * kVec, a.cols);
                const bool there = col + s * kSlice < a.cols;
                load_row<0>(d[s], a.dy, token, a.cols, there, l[s]);
                load_row<0>(t[s], a.table, row, a.cols, there, l[s]);
            }
#pragma unroll
            for (int s = 0; s < kSlices; ++s) {
                settle(d[s], l[s], a.cols);
                settle(t[s], l[s], a.cols);
#pragma unroll
                for (int i = 0; i < kVec; ++i) sum = fmaf(d[s][i], t[s][i], sum);
            }
        }
        sum = wave_sum(sum) * a.scale;
    }
    if (lane == 0) store1(a.dweights.data, a.dweights.dtype, p, sum);
}
template <class D, class T>
__global__ __launch_bounds__(kThreads) void apm_lookup_weights_kernel(WeightGradArgs a, uint32_t first) {
    const uint32_t p = first + blockIdx.x * kWaves + (uint32_t)__builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    if (p < a.n) weight_grad<D, T>(a, p, (int)threadIdx.x % kWave);
}

// ---- the gradient of the table ------------------------------------------------------------------
constexpr int kChunkMost = kWave;           // sorted positions of a wavefront, one of each lane to begin with
constexpr int kChunkLeast = 8;
constexpr int kAhead = 8;                   // rows of dy under way
constexpr int kEmptyRows = 8;              // rows of dtable that a wavefront looks through for those without positions

struct TableGradArgs {
    const void* ids;
    const int32_t* order;
    const int64_t* offsets;
    float* parts;  // [chunks][2][cols_8]: of the row that began before the chunk, and of the row that goes on behind it
    u32x2* on;     // [chunks]: the row that begins in the chunk and goes on behind it, and how many chunks have parts of it; 0 of no row
    apm_matrix dy, dtable;
    apm_vector weights;
    uint32_t n, rows, per_token, chunk, chunks, slices, empty;  // empty: wavefronts that write zeros
    uint32_t first_item, last_item;
    int32_t cols, cols_8, id_type, accumulate;
    float scale;
};

template <class T> __device__ __forceinline__ void finish_row(const TableGradArgs& a, uint32_t row, const LaneCols& l, float (&v)[kVec]) {
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] *= a.scale;
    if (a.accumulate) {
        Raw<T> old;
        load_row(old, a.dtable, row, a.cols, true, l);
        settle(old, l, a.cols);
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] += old[i];
    }
    store_row<T, 0>(a.dtable, row, a.cols, true, l, v);
}
__device__ __forceinline__ float* part_of(const TableGradArgs& a, uint32_t chunk, int which, int col) {
    return a.parts + ((uint64_t)chunk * 2 + (uint32_t)which) * (uint32_t)a.cols_8 + (uint32_t)col;
}
__device__ __forceinline__ uint32_t row_at(const TableGradArgs& a, uint32_t i) {
    const uint32_t p = (uint32_t)a.order[i];
    return p < a.n ? row_of(a.ids, a.id_type, p, a.rows) : a.rows;
}

// 16384 positions of a 50257 x 2048 table in bf16: 49 us = 5.6 TB/s of what has to move, three quarters of which are zeros, for which a fill of that size takes 30.
// Zeros are stored non-temporally (56 us without), sums are not (53.7 with).
// W: of the table, if the gradient of the weights is made by the same launch; void: it is not.
template <class D, class T, class W>
__global__ __launch_bounds__(kThreads) void apm_table_grad_kernel(TableGradArgs a, WeightGradArgs of_weights) {
    const int lane = (int)threadIdx.x % kWave;
    const uint32_t item = a.first_item + (uint32_t)__builtin_amdgcn_readfirstlane((int)(blockIdx.x * kWaves + threadIdx.x / kWave));
    const uint32_t summing = a.chunks * a.slices;
    LaneCols l;
    if (item >= summing) {  // rows without positions
        const uint32_t e = item - summing;
        if (e >= a.empty) {
            if constexpr (!std::is_void<W>::value) {
                if (e - a.empty < of_weights.n) weight_grad<D, W>(of_weights, e - a.empty, lane);
            }
            return;
        }
        const uint32_t first = e * kEmptyRows, r = first + (uint32_t)lane;
        const bool none = lane < kEmptyRows && r < a.rows && a.offsets[r] >= a.offsets[r + 1];
        uint64_t mask = __ballot(none);
        const float zero[kVec] = {};
        while (mask) {
            const uint32_t row = first + (uint32_t)__builtin_ctzll(mask);
            mask &= mask - 1;
            for (int col = 0; col < a.cols; col += kSlice) {
                l.set(col + lane * kVec, a.cols);
                store_row<T>(a.dtable, row, a.cols, true, l, zero);
            }
        }
        return;
    }
    const uint32_t chunk = item / a.slices, start = chunk * a.chunk;
    const int n = (int)min(a.chunk, a.n - start);
    l.set((int)(item - chunk * a.slices) * kSlice + lane * kVec, a.cols);
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
    const bool notes = item == chunk * a.slices && lane == 0;
    uint32_t row = of_lane(my_row, 0);
    if (row >= a.rows) {  // so are all behind it
        if (notes) a.on[chunk] = u32x2{0u, 0u};
        return;
    }
    bool before = start > 0 && row_at(a, start - 1) == row;  // the row began in an earlier chunk
    const uint32_t next = start + a.chunk, after = next < a.n ? row_at(a, next) : a.rows;
    const int64_t end = min(max(a.offsets[min(after, a.rows - 1) + 1], (int64_t)next + 1), (int64_t)a.n);  // of `after`, if it is a row
    float sum[kVec] = {};
    auto flush = [&](bool goes_on) {
        if (!before && !goes_on) return finish_row<T>(a, row, l, sum);
        if (l.n <= 0) return;
        u32x4 w[2];
#pragma unroll
        for (int i = 0; i < kVec; ++i) w[i / 4][i % 4] = __builtin_bit_cast(uint32_t, sum[i]);
        u32x4* to = (u32x4*)part_of(a, chunk, before ? 0 : 1, l.col);
        to[0] = w[0], to[1] = w[1];
    };
    for (int i0 = 0; i0 < n; i0 += kAhead) {
        Raw<D> x[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int i = i0 + k;
            const bool in = i < n && of_lane(my_row, i & (kWave - 1)) < a.rows;
            load_row(x[k], a.dy, of_lane(my_token, i & (kWave - 1)), a.cols, in, l);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int i = i0 + k;
            if (i >= n) break;
            const uint32_t r = of_lane(my_row, i);
            if (r != row) {
                flush(false);
                if (r >= a.rows) {
                    if (notes) a.on[chunk] = u32x2{0u, 0u};
                    return;
                }
                row = r, before = false;
#pragma unroll
                for (int e = 0; e < kVec; ++e) sum[e] = 0.0f;
            }
            const float w = of_lane(my_weight, i);
            settle(x[k], l, a.cols);
#pragma unroll
            for (int e = 0; e < kVec; ++e) sum[e] = fmaf(w, x[k][e], sum[e]);
        }
    }
    flush(after == row);
    if (notes) a.on[chunk] = u32x2{row, after == row && !before ? (uint32_t)(end - 1) / a.chunk - chunk + 1 : 0u};
}

// A row that goes beyond the chunk in which it begins: that chunk's part and those of the chunks behind it.  Each wavefront looks at what a chunk noted; what there is
// to do, which is little, the workgroup does together, a stretch of the parts for each wavefront.  6.4 us for the embedding above: launch, the note, and the longest
// row's 72 parts (7.9 where the order was looked at anew, three loads one after the other).
constexpr int kPartsAhead = 8;
template <class T>
__global__ __launch_bounds__(kThreads) void apm_table_grad_join_kernel(TableGradArgs a) {
    __shared__ float sums[kWaves][kVec][kWave];
    __shared__ uint32_t rows[kWaves], parts_of[kWaves];
    const int lane = (int)threadIdx.x % kWave;
    const uint32_t wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    auto item_of = [&](uint32_t w) { return a.first_item + blockIdx.x + w * gridDim.x; };  // neighbours, which may have the same row's slices, are for different workgroups
    {
        const uint32_t item = item_of(wave);
        const u32x2 on = item < a.last_item ? a.on[item / a.slices] : u32x2{0u, 0u};
        const uint32_t row = on.x, parts = on.y;
        if (lane == 0) rows[wave] = row, parts_of[wave] = parts;
    }
    __syncthreads();
    for (uint32_t w = 0; w < kWaves; ++w) {
        const uint32_t parts = (uint32_t)__builtin_amdgcn_readfirstlane((int)parts_of[w]), row = (uint32_t)__builtin_amdgcn_readfirstlane((int)rows[w]);
        if (parts == 0) continue;
        const uint32_t chunk = item_of(w) / a.slices, each = (parts + kWaves - 1) / kWaves, from = min(wave * each, parts), to = min(from + each, parts);
        LaneCols l;
        l.set((int)(item_of(w) - chunk * a.slices) * kSlice + lane * kVec, a.cols);
        float sum[kVec] = {};
        for (uint32_t c = from; c < to; c += kPartsAhead) {
            Raw<float> x[kPartsAhead];
#pragma unroll
            for (int k = 0; k < kPartsAhead; ++k) {
                const uint32_t i = min(c + (uint32_t)k, to - 1);
                x[k].load(part_of(a, chunk + i, i == 0 ? 1 : 0, 0), l.col, c + (uint32_t)k < to && l.n > 0 ? kVec : 0);
            }
#pragma unroll
            for (int k = 0; k < kPartsAhead; ++k)
#pragma unroll
                for (int i = 0; i < kVec; ++i) sum[i] += x[k][i];
        }
#pragma unroll
        for (int i = 0; i < kVec; ++i) sums[wave][i][lane] = sum[i];
        __syncthreads();
        if (wave == 0) {
#pragma unroll
            for (int v = 1; v < kWaves; ++v)
#pragma unroll
                for (int i = 0; i < kVec; ++i) sum[i] += sums[v][i][lane];
            finish_row<T>(a, row, l, sum);
        }
        __syncthreads();
    }
}

// Positions of a wavefront: few, so that there are wavefronts for the whole chip, but no more of them than that, since rows that go beyond a chunk are
// written and read once more (the embedding above with chunks for 2048, 4096 and 8192 wavefronts, both kernels: 61.5, 61.6, 71 us when this was chosen).
constexpr int64_t kChunksWanted = 4096;
int64_t chunk_of(const apm_lookup& l) {
    const int64_t n = l.tokens * l.per_token, slices = div_up(l.cols, kSlice);
    if (n <= kChunkMost / 2) return kChunkMost / 2;  // one chunk needs no second kernel
    int64_t chunk = kChunkLeast;
    while (chunk < kChunkMost && div_up(n, chunk) * slices > kChunksWanted) chunk *= 2;
    return chunk;
}
size_t parts_of(const apm_lookup& l) { return (size_t)div_up(l.tokens * l.per_token, chunk_of(l)) * 2 * (size_t)div_up(l.cols, kVec) * kVec; }
size_t room_of(const apm_lookup& l) { return parts_of(l) * sizeof(float) + (size_t)div_up(l.tokens * l.per_token, chunk_of(l)) * sizeof(u32x2); }

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
    const int64_t most_items = workgroups_of_launch(kThreads) * kWaves;  // whole workgroups: what one has to spare would be the next launch's, whose rows are added once
    const bool wide_dy = n > 0 && g.dy.dtype == APM_F32, wide_dtable = g.dtable.dtype == APM_F32, wide_table = l.table.dtype == APM_F32;
    WeightGradArgs of_weights{};
    of_weights.ids = l.ids.data, of_weights.id_type = l.ids.type, of_weights.dy = g.dy, of_weights.table = l.table, of_weights.dweights = g.dweights;
    of_weights.n = (uint32_t)n, of_weights.per_token = (uint32_t)l.per_token, of_weights.cols = (int32_t)l.cols, of_weights.rows = (uint32_t)l.rows;
    of_weights.scale = (float)l.scale;
    bool weights = g.dweights.data && n > 0;
    if (g.dtable.data) {
        TableGradArgs a{};
        a.ids = l.ids.data, a.id_type = l.ids.type, a.dy = g.dy, a.dtable = g.dtable, a.order = g.order, a.offsets = g.offsets;
        a.parts = (float*)workspace, a.on = (u32x2*)(a.parts + parts_of(l)), a.weights = l.weights;
        a.n = (uint32_t)n, a.rows = (uint32_t)l.rows, a.per_token = (uint32_t)l.per_token, a.cols = (int32_t)l.cols, a.cols_8 = (int32_t)(div_up(l.cols, kVec) * kVec);
        a.chunk = (uint32_t)chunk_of(l), a.chunks = (uint32_t)div_up(n, a.chunk), a.slices = (uint32_t)div_up(l.cols, kSlice), a.empty = g.accumulate ? 0 : (uint32_t)div_up(l.rows, kEmptyRows);
        a.accumulate = g.accumulate, a.scale = (float)l.scale;
        const int64_t summing = (int64_t)a.chunks * a.slices;
        if (summing + a.empty > INT32_MAX) return fail(APM_EINVAL, "too many positions for so many columns");
        const bool both = weights && summing + a.empty + n <= most_items;  // by one launch
        const int64_t items = summing + a.empty + (both ? n : 0);
        for (int64_t at = 0; at < items; at += most_items) {
            a.first_item = (uint32_t)at;
            const dim3 grid((unsigned)div_up(std::min(most_items, items - at), kWaves)), block(kThreads);
            auto start = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, s, a, of_weights); };
            auto with = [&](auto d, auto t) {
                typedef decltype(d) D;
                typedef decltype(t) T;
                if (!both) start(apm_table_grad_kernel<D, T, void>);
                else if (wide_table) start(apm_table_grad_kernel<D, T, float>);
                else start(apm_table_grad_kernel<D, T, bf16>);
            };
            if (wide_dy) wide_dtable ? with(float(), float()) : with(float(), bf16());
            else wide_dtable ? with(bf16(), float()) : with(bf16(), bf16());
            APM_HIP(hipGetLastError());
        }
        if (both) weights = false;
        if (a.chunks > 1) {
            for (int64_t at = 0; at < summing; at += most_items) {
                a.first_item = (uint32_t)at, a.last_item = (uint32_t)std::min(summing, at + most_items);
                const dim3 grid((unsigned)div_up(a.last_item - at, kWaves)), block(kThreads);
                if (wide_dtable) hipLaunchKernelGGL(apm_table_grad_join_kernel<float>, grid, block, 0, s, a);
                else hipLaunchKernelGGL(apm_table_grad_join_kernel<bf16>, grid, block, 0, s, a);
                APM_HIP(hipGetLastError());
            }
        }
    }
    if (weights) {
        for (int64_t at = 0; at < n; at += most_items) {
            const dim3 grid((unsigned)div_up(std::min(most_items, n - at), kWaves)), block(kThreads);
            auto start = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, s, of_weights, (uint32_t)at); };
            if (wide_dy) wide_table ? start(apm_lookup_weights_kernel<float, float>) : start(apm_lookup_weights_kernel<float, bf16>);
            else wide_table ? start(apm_lookup_weights_kernel<bf16, float>) : start(apm_lookup_weights_kernel<bf16, bf16>);
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
