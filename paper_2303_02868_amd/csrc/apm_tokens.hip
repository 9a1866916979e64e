// Positions sorted by their ids, stably: digits of eight bits from the lowest on.  What is sorted is a key for each position, its id or `rows` where that is no
// row, so that those come last.
//
// Few positions (up to kOnePositions) are sorted by one workgroup in LDS, where a pass costs two barriers and no launch.  More of them: each pass counts the digits of
// each tile of positions, and then each tile adds up what stands before it and puts its positions where they belong.
#include <algorithm>

#include "apm_tok.h"

namespace apm {
namespace {

constexpr int kDigitBits = 8, kDigits = 1 << kDigitBits, kWave = 64;

struct SortArgs {
    const void* ids;
    int32_t* order;
    int64_t* offsets;
    int32_t* place;
    int32_t* token;
    uint32_t n, rows, passes;
    uint32_t per_token;
    int32_t id_type;
    int32_t alone;  // the one workgroup writes offsets, too
};

// Lanes of the wavefront with the same digit as this one, among those that are there.
__device__ __forceinline__ uint64_t same_digit(uint32_t digit, bool there) {
    uint64_t mask = __ballot(there);
#pragma unroll
    for (int b = 0; b < kDigitBits; ++b) {
        const uint64_t set = __ballot((digit >> b) & 1u);
        mask &= (digit >> b) & 1u ? set : ~set;
    }
    return mask;
}
__device__ __forceinline__ uint32_t lanes_below(uint64_t mask) {
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0u));
}

// What precedes each of 256 numbers, which the first 256 threads hold (all threads of the workgroup take part).
__device__ __forceinline__ uint32_t before_among_digits(uint32_t v, uint32_t* of_waves) {
    const int lane = (int)threadIdx.x % kWave, wave = (int)threadIdx.x / kWave;
    uint32_t up = v;
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
        const uint32_t o = __shfl_up(up, d);
        if (lane >= d) up += o;
    }
    if (wave < kDigits / kWave && lane == kWave - 1) of_waves[wave] = up;
    __syncthreads();
    uint32_t before = up - v;
    for (int w = 0; w < min(wave, kDigits / kWave); ++w) before += of_waves[w];
    return before;
}

__device__ __forceinline__ void put(const SortArgs& a, uint32_t i, uint32_t p, uint32_t key) {
    a.order[i] = (int32_t)p;
    if (a.place) a.place[p] = key < a.rows ? (int32_t)i : -1;
    if (a.token) a.token[i] = (int32_t)(p / a.per_token);
}
// The first of n sorted keys that is `row` or larger.
template <class Key> __device__ __forceinline__ uint32_t first_of(const Key* keys, uint32_t n, uint32_t row) {
    uint32_t lo = 0, hi = n;
    while (lo < hi) {
        const uint32_t mid = (lo + hi) / 2;
        if (keys[mid] < row) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

// ---- one workgroup ------------------------------------------------------------------------------
// Positions lie in LDS in the order of the passes so far, each wavefront takes a stretch of them into registers: counts of each digit in each
// stretch, what stands before, and back to LDS in the new order.
constexpr int kOneThreads = 1024, kOneWaves = kOneThreads / kWave, kOneMost = 16;  // positions of a thread
constexpr uint32_t kOnePositions = kOneThreads * kOneMost;
template <int PER>
__global__ __launch_bounds__(kOneThreads) void apm_sort_one_kernel(SortArgs a, uint32_t* sorted) {
    constexpr uint32_t kMost = kOneThreads * PER;
    __shared__ uint32_t keys[kMost];
    __shared__ uint16_t at[kMost];
    __shared__ uint32_t counts[kOneWaves][kDigits];
    __shared__ uint32_t of_waves[kDigits / kWave];
    const int tid = (int)threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    const uint32_t n = a.n, first = (uint32_t)wave * (PER * kWave);
    uint32_t key[PER], pos[PER];
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        pos[u] = first + (uint32_t)(u * kWave + lane);
        key[u] = pos[u] < n ? row_of(a.ids, a.id_type, pos[u], a.rows) : 0u;
    }
    for (uint32_t pass = 0; pass < a.passes; ++pass) {
        const uint32_t shift = pass * kDigitBits;
        for (int i = tid; i < kOneWaves * kDigits; i += kOneThreads) (&counts[0][0])[i] = 0;
        __syncthreads();
        uint32_t rank[PER];  // among the stretch's of the same digit
#pragma unroll
        for (int u = 0; u < PER; ++u) {
            const uint32_t i = first + (uint32_t)(u * kWave + lane), digit = (key[u] >> shift) & (kDigits - 1);
            const bool there = i < n;
            if (first + (uint32_t)(u * kWave) >= n) continue;
            const uint64_t same = same_digit(digit, there);
            const uint32_t below = lanes_below(same);
            uint32_t seen = 0;
            if (there) seen = counts[wave][digit];
            rank[u] = seen + below;
            among_lanes();
            if (there && below == 0) counts[wave][digit] = seen + (uint32_t)__popcll(same);
            among_lanes();
        }
        __syncthreads();
        uint32_t total = 0;
        if (tid < kDigits) {
#pragma unroll
            for (int w = 0; w < kOneWaves; ++w) {
                const uint32_t c = counts[w][tid];
                counts[w][tid] = total;
                total += c;
            }
        }
        const uint32_t before = before_among_digits(total, of_waves);
        if (tid < kDigits) {
#pragma unroll
            for (int w = 0; w < kOneWaves; ++w) counts[w][tid] += before;
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < PER; ++u) {
            const uint32_t i = first + (uint32_t)(u * kWave + lane);
            if (i >= n) continue;
            const uint32_t to = counts[wave][(key[u] >> shift) & (kDigits - 1)] + rank[u];
            keys[to] = key[u];
            at[to] = (uint16_t)pos[u];
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < PER; ++u) {
            const uint32_t i = first + (uint32_t)(u * kWave + lane);
            key[u] = i < n ? keys[i] : 0u;
            pos[u] = i < n ? at[i] : i;
        }
    }
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        const uint32_t i = first + (uint32_t)(u * kWave + lane);
        if (i >= n) continue;
        put(a, i, pos[u], key[u]);
        if (!a.alone) sorted[i] = key[u];
    }
    if (a.offsets && a.alone)
        for (uint32_t r = (uint32_t)tid; r <= a.rows; r += kOneThreads) a.offsets[r] = first_of(keys, n, r);
}

// ---- many workgroups ----------------------------------------------------------------------------
constexpr int kManyThreads = 256, kManyWaves = kManyThreads / kWave;

struct PassArgs {
    const uint32_t* keys;  // nullptr: the ids, positions in their order
    const int32_t* at;
    uint32_t* keys_out;    // nullptr: not needed any more
    int32_t* at_out;       // nullptr: the last pass
    uint32_t* counts;      // [tiles][digits]
    uint32_t shift, tile, tiles;
};
__device__ __forceinline__ uint32_t key_of(const SortArgs& a, const PassArgs& s, uint32_t i) {
    return s.keys ? s.keys[i] : row_of(a.ids, a.id_type, i, a.rows);
}

__global__ __launch_bounds__(kManyThreads) void apm_sort_count_kernel(SortArgs a, PassArgs s) {
    __shared__ uint32_t counts[kDigits];
    counts[threadIdx.x] = 0;
    __syncthreads();
    const uint32_t begin = blockIdx.x * s.tile, end = (uint32_t)min((uint64_t)a.n, (uint64_t)begin + s.tile);
#pragma unroll 4
    for (uint32_t i = begin + threadIdx.x; i < end; i += kManyThreads) atomicAdd(&counts[(key_of(a, s, i) >> s.shift) & (kDigits - 1)], 1u);
    __syncthreads();
    s.counts[(uint64_t)blockIdx.x * kDigits + threadIdx.x] = counts[threadIdx.x];
}

__global__ __launch_bounds__(kManyThreads) void apm_sort_place_kernel(SortArgs a, PassArgs s) {
    static_assert(kManyThreads == kDigits, "a thread has a digit");
    __shared__ uint32_t next[kManyWaves][kDigits];
    __shared__ uint32_t of_waves[kDigits / kWave];
    const int tid = (int)threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    uint32_t all = 0, mine = 0;  // positions with the thread's digit: of all tiles, of those before this one
#pragma unroll 8
    for (uint32_t t = 0; t < s.tiles; ++t) {
        const uint32_t c = s.counts[(uint64_t)t * kDigits + (uint32_t)tid];
        if (t < blockIdx.x) mine += c;
        all += c;
    }
    const uint32_t before = before_among_digits(all, of_waves);
    // One pass sorts all, and its digits are the rows: their counts are the offsets.
    if (a.offsets && a.passes == 1 && blockIdx.x == 0 && (uint32_t)tid <= a.rows) a.offsets[tid] = before;
    const uint32_t begin = blockIdx.x * s.tile, end = (uint32_t)min((uint64_t)a.n, (uint64_t)begin + s.tile), each = s.tile / kManyWaves;
    const uint32_t from = (uint32_t)min((uint64_t)begin + (uint64_t)wave * each, (uint64_t)end), to = (uint32_t)min((uint64_t)from + each, (uint64_t)end);
#pragma unroll
    for (int w = 0; w < kManyWaves; ++w) next[w][tid] = 0;
    __syncthreads();
    for (uint32_t i = from + (uint32_t)lane; i < to; i += kWave) atomicAdd(&next[wave][(key_of(a, s, i) >> s.shift) & (kDigits - 1)], 1u);
    __syncthreads();
    uint32_t sum = before + mine;
#pragma unroll
    for (int w = 0; w < kManyWaves; ++w) {
        const uint32_t c = next[w][tid];
        next[w][tid] = sum;
        sum += c;
    }
    __syncthreads();
    for (uint32_t base = from; base < to; base += kWave) {
        const uint32_t i = base + (uint32_t)lane;
        const bool there = i < to;
        const uint32_t key = there ? key_of(a, s, i) : 0u, digit = (key >> s.shift) & (kDigits - 1), p = there && s.at ? (uint32_t)s.at[i] : i;
        const uint64_t same = same_digit(digit, there);
        const uint32_t below = lanes_below(same);
        uint32_t at = 0;
        if (there) at = next[wave][digit] + below;
        among_lanes();
        if (there && below == 0) next[wave][digit] = at + (uint32_t)__popcll(same);
        among_lanes();
        if (!there) continue;
        if (s.keys_out) s.keys_out[at] = key;
        if (s.at_out) s.at_out[at] = (int32_t)p;
        else put(a, at, p, key);
    }
}

// offsets where the sorted keys are in memory: each row looks for its first.
constexpr int kOffsetThreads = 256;
__global__ __launch_bounds__(kOffsetThreads) void apm_sort_offsets_kernel(const uint32_t* keys, uint32_t n, uint32_t rows, int64_t* offsets) {
    const uint32_t r = blockIdx.x * kOffsetThreads + threadIdx.x;
    if (r <= rows) offsets[r] = first_of(keys, n, r);
}

constexpr int64_t kTilesMost = 512, kTileLeast = 4096;
constexpr uint32_t kOneRows = 4096;  // offsets of so many rows are written by the one workgroup

struct SortShape {
    bool one;
    uint32_t passes, tile, tiles;
};
SortShape sort_shape(int64_t n, int64_t rows) {
    SortShape s{};
    uint32_t bits = 1;
    while ((rows >> bits) != 0) ++bits;  // keys are 0 .. rows
    s.passes = (bits + kDigitBits - 1) / kDigitBits;
    s.one = n <= kOnePositions;
    const int64_t tile = std::max(kTileLeast, div_up(div_up(n, kTilesMost), kTileLeast) * kTileLeast);
    s.tile = (uint32_t)tile, s.tiles = (uint32_t)div_up(n, tile);
    return s;
}
size_t to_16(size_t bytes) { return (bytes + 15) / 16 * 16; }
size_t room_of(int64_t n, int64_t rows) {
    const SortShape s = sort_shape(n, rows);
    const size_t words = to_16((size_t)n * 4);
    if (s.one) return words;
    return (size_t)s.tiles * kDigits * 4 + 4 * words;  // keys and positions, of two passes
}

int check_order(const apm_token_order& o) {
    if (o.n < 0 || o.n > APM_MAX_POSITIONS || o.rows < 1 || o.rows > APM_MAX_POSITIONS || o.per_token < 1 || o.per_token > APM_MAX_POSITIONS)
        return fail(APM_EINVAL, "bad size: %lld positions, %lld of a token, %lld rows", (long long)o.n, (long long)o.per_token, (long long)o.rows);
    if (o.n > 0) {
        const int rc = check_indices("ids", o.ids);
        if (rc != APM_OK) return rc;
        if (!o.order) return fail(APM_EINVAL, "order is missing");
    }
    if (!aligned_to(o.order, 4) || !aligned_to(o.place, 4) || !aligned_to(o.token, 4) || !aligned_to(o.offsets, 8))
        return fail(APM_EINVAL, "order, place, token or offsets are not aligned to their elements");
    return APM_OK;
}

int sort_tokens(const apm_token_order* op, void* workspace, size_t workspace_bytes, void* stream) {
    if (!op) return fail(APM_EINVAL, "missing argument");
    const apm_token_order& o = *op;
    int rc = check_order(o);
    if (rc == APM_OK) rc = check_room(workspace, workspace_bytes, room_of(o.n, o.rows));
    if (rc != APM_OK) return rc;
    const SortShape shape = sort_shape(o.n, o.rows);
    SortArgs a{};
    a.ids = o.ids.data, a.id_type = o.ids.type;
    a.order = o.order, a.offsets = o.offsets, a.place = o.place, a.token = o.token;
    a.n = (uint32_t)o.n, a.rows = (uint32_t)o.rows, a.per_token = (uint32_t)o.per_token, a.passes = shape.passes;
    const hipStream_t st = (hipStream_t)stream;
    const uint32_t* sorted = nullptr;
    bool search = false;  // offsets have still to be found, in the sorted keys
    if (shape.one) {
        a.alone = !o.offsets || a.rows <= kOneRows;
        sorted = (const uint32_t*)workspace, search = !a.alone;
        auto start = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(1), dim3(kOneThreads), 0, st, a, (uint32_t*)workspace); };
        if (a.n <= kOneThreads) start(apm_sort_one_kernel<1>);
        else if (a.n <= 4 * kOneThreads) start(apm_sort_one_kernel<4>);
        else start(apm_sort_one_kernel<kOneMost>);
        APM_HIP(hipGetLastError());
    } else {
        char* room = (char*)workspace;
        const size_t words = to_16((size_t)o.n * 4);
        uint32_t* counts = (uint32_t*)room;
        room += (size_t)shape.tiles * kDigits * 4;
        uint32_t* keys[2] = {(uint32_t*)room, (uint32_t*)(room + words)};
        int32_t* at[2] = {(int32_t*)(room + 2 * words), (int32_t*)(room + 3 * words)};
        for (uint32_t pass = 0; pass < shape.passes; ++pass) {
            const bool last = pass + 1 == shape.passes;
            PassArgs s{};
            s.keys = pass > 0 ? keys[(pass - 1) % 2] : nullptr, s.at = pass > 0 ? at[(pass - 1) % 2] : nullptr;
            s.keys_out = !last || (o.offsets && pass > 0) ? keys[pass % 2] : nullptr, s.at_out = last ? nullptr : at[pass % 2];
            s.counts = counts, s.shift = pass * kDigitBits, s.tile = shape.tile, s.tiles = shape.tiles;
            hipLaunchKernelGGL(apm_sort_count_kernel, dim3(shape.tiles), dim3(kManyThreads), 0, st, a, s);
            hipLaunchKernelGGL(apm_sort_place_kernel, dim3(shape.tiles), dim3(kManyThreads), 0, st, a, s);
            APM_HIP(hipGetLastError());
            if (last) sorted = s.keys_out, search = o.offsets && pass > 0;
        }
    }
    if (search) {
        hipLaunchKernelGGL(apm_sort_offsets_kernel, dim3((unsigned)div_up(o.rows + 1, kOffsetThreads)), dim3(kOffsetThreads), 0, st, sorted, a.n, a.rows, o.offsets);
        APM_HIP(hipGetLastError());
    }
    return APM_OK;
}

}  // namespace
}  // namespace apm

extern "C" size_t apm_sort_tokens_workspace_bytes(const apm_token_order* o) {
    return !o || apm::check_order(*o) != APM_OK ? 0 : apm::room_of(o->n, o->rows);
}

extern "C" int apm_sort_tokens(const apm_token_order* o, void* workspace, size_t workspace_bytes, void* stream) {
    return apm::guarded([&]() -> int { return apm::sort_tokens(o, workspace, workspace_bytes, stream); });
}
