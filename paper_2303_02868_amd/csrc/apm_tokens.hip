// Positions sorted by their ids, stably: digits of eight bits from the lowest on.  What is sorted is a key for each position, its id or `rows` where that is no
// row, so that those come last.
//
// All latency: 16384 positions are 0.7 MB.  Few positions (up to kOnePositions) are sorted by one workgroup in LDS, where a pass costs four barriers and no launch
// (16 positions 3.0 us, 4000 words 12.7).  More of them: each pass counts the digits of each tile of positions, and then each tile adds up what stands before it and puts its
// positions where they belong (16384 words 19.8 us; by one workgroup 35, by tiles that count everything for themselves 24.7; 32768, 65536 and 131072 words 20, 23.5 and 27).
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
constexpr int kOneThreads = 1024, kOneWaves = kOneThreads / kWave, kOneMost = 4;  // positions of a thread
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
    if (!a.offsets || !a.alone) return;
    // offsets[r] = i for the rows r behind the key in front of i, up to the key at i; those behind the last key belong to i = n.  A wavefront goes through its
    // positions' stretches: short ones a lane each, longer ones together.
    constexpr uint32_t kShort = 4;
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        const uint32_t i = first + (uint32_t)(u * kWave + lane);
        uint32_t row = 0, stretch = 0;
        if (i <= n && i < kMost) {
            const uint32_t last = i < n ? key[u] : a.rows;
            row = i > 0 ? keys[i - 1] + 1 : 0;
            stretch = last + 1 - row;
        }
        for (uint32_t k = 0; k < kShort; ++k)
            if (k < stretch && stretch <= kShort) a.offsets[row + k] = i;
        uint64_t longer = __ballot(stretch > kShort);
        while (longer) {
            const int l = __builtin_ctzll(longer);
            longer &= longer - 1;
            const uint32_t from = (uint32_t)__builtin_amdgcn_readlane((int)row, l), count = (uint32_t)__builtin_amdgcn_readlane((int)stretch, l), at = first + (uint32_t)(u * kWave + l);
            for (uint32_t k = (uint32_t)lane; k < count; k += kWave) a.offsets[from + k] = at;
        }
    }
    if (n == kMost) {
        for (uint32_t r = keys[n - 1] + 1 + (uint32_t)tid; r <= a.rows; r += kOneThreads) a.offsets[r] = n;
    }
}

// ---- many workgroups ----------------------------------------------------------------------------
constexpr int kManyThreads = 1024, kManyWaves = kManyThreads / kWave;

struct PassArgs {
    const uint32_t* keys;  // nullptr: the ids, positions in their order
    const int32_t* at;
    uint32_t* keys_out;    // nullptr: not needed any more
    int32_t* at_out;       // nullptr: the last pass
    uint32_t* counts;      // [tiles][digits], and of the passes behind this one behind it
    uint32_t shift, tile, tiles;
    uint32_t behind;       // passes whose counts are the placing kernel's
};
__device__ __forceinline__ uint32_t key_of(const SortArgs& a, const PassArgs& s, uint32_t i) {
    return s.keys ? s.keys[i] : row_of(a.ids, a.id_type, i, a.rows);
}

// Adds the wavefront's digits to counts in LDS.  Keys that earlier passes have put side by side are often equal, and additions to one place come one after the
// other: the first lane of a run of equal digits adds the whole run (16384 words, the second pass: 15 us each for itself, so 7).
__device__ __forceinline__ void count(uint32_t* counts, uint32_t digit, bool there) {
    const uint32_t lane = threadIdx.x % kWave, left = (uint32_t)__shfl_up((int)digit, 1);
    const uint64_t in = __ballot(there), first = __ballot(there && (lane == 0 || left != digit));
    if (!((first >> lane) & 1)) return;
    const uint64_t above = lane == kWave - 1 ? 0 : first >> (lane + 1);
    const uint32_t next = above ? lane + 1 + (uint32_t)__builtin_ctzll(above) : (uint32_t)__popcll(in);  // lanes that are there are the first ones
    atomicAdd(&counts[digit], next - lane);
}

__global__ __launch_bounds__(kManyThreads) void apm_sort_count_kernel(SortArgs a, PassArgs s) {
    __shared__ uint32_t counts[kDigits];
    const uint32_t begin = blockIdx.x * s.tile, end = (uint32_t)min((uint64_t)a.n, (uint64_t)begin + s.tile);
    uint32_t key = key_of(a, s, min(begin + threadIdx.x, end - 1));
    if (threadIdx.x < kDigits) counts[threadIdx.x] = 0;
    __syncthreads();
    for (uint32_t base = begin; base < end; base += kManyThreads) {
        count(counts, (key >> s.shift) & (kDigits - 1), base + threadIdx.x < end);
        if (base + kManyThreads < end) key = key_of(a, s, min(base + kManyThreads + threadIdx.x, end - 1));
    }
    __syncthreads();
    if (threadIdx.x >= kDigits) return;
    for (uint32_t pass = 0; pass <= s.behind; ++pass) s.counts[((uint64_t)pass * s.tiles + blockIdx.x) * kDigits + threadIdx.x] = pass == 0 ? counts[threadIdx.x] : 0;
}

// ONCE: a tile is a position for each thread.  TALLY: of few tiles, and where a position goes is counted for the next pass, too, in LDS and then in memory, by additions of
// whole numbers, whose order does not matter (a kernel less; 16384 words 22.0 us, so 19.8, 5000 19.9 and 17).  Otherwise each wavefront goes through its stretch twice, to count it and to put it in place.
constexpr uint32_t kTallied = 32;  // tiles
template <bool ONCE, bool TALLY>
__global__ __launch_bounds__(kManyThreads) void apm_sort_place_kernel(SortArgs a, PassArgs s) {
    static_assert(ONCE || !TALLY, "a position for each thread");
    __shared__ uint32_t tally[TALLY ? kTallied * kDigits : 1];
    __shared__ uint32_t next[kManyWaves][kDigits];
    __shared__ uint32_t seen[2][kDigits];  // positions with a digit: of the tiles before this one, of the others
    __shared__ uint32_t of_waves[kDigits / kWave];
    const int tid = (int)threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    const uint32_t begin = blockIdx.x * s.tile, end = (uint32_t)min((uint64_t)a.n, (uint64_t)begin + s.tile), each = s.tile / kManyWaves;
    const uint32_t from = (uint32_t)min((uint64_t)begin + (uint64_t)wave * each, (uint64_t)end), to = (uint32_t)min((uint64_t)from + each, (uint64_t)end);
    auto key_at = [&](uint32_t i) { return i < to ? key_of(a, s, i) : 0u; };
    auto position_at = [&](uint32_t i) { return s.at && i < to ? (uint32_t)s.at[i] : i; };
    const uint32_t key0 = key_at(from + (uint32_t)lane), p0 = position_at(from + (uint32_t)lane);
    uint32_t sum[2] = {0, 0};
    constexpr uint32_t kParts = kManyThreads / kDigits;
#pragma unroll 8
    for (uint32_t t = (uint32_t)tid / kDigits; t < s.tiles; t += kParts) {
        const uint32_t c = s.counts[(uint64_t)t * kDigits + (uint32_t)tid % kDigits];
        sum[0] += t < blockIdx.x ? c : 0;
        sum[1] += t < blockIdx.x ? 0 : c;
    }
    for (int i = tid; i < kManyWaves * kDigits; i += kManyThreads) (&next[0][0])[i] = 0;
    if (tid < 2 * kDigits) (&seen[0][0])[tid] = 0;
    if constexpr (TALLY)
        for (uint32_t i = (uint32_t)tid; i < s.tiles * kDigits; i += kManyThreads) tally[i] = 0;
    __syncthreads();
    uint64_t same = 0;
    uint32_t below = 0;
    if constexpr (ONCE) {
        const uint32_t digit = (key0 >> s.shift) & (kDigits - 1);
        const bool there = from + (uint32_t)lane < to;
        same = same_digit(digit, there), below = lanes_below(same);
        if (there && below == 0) next[wave][digit] = (uint32_t)__popcll(same);
    } else {
        for (uint32_t base = from; base < to; base += kWave) count(next[wave], (key_at(base + (uint32_t)lane) >> s.shift) & (kDigits - 1), base + (uint32_t)lane < to);
    }
    atomicAdd(&seen[0][tid % kDigits], sum[0]);
    atomicAdd(&seen[1][tid % kDigits], sum[1]);
    __syncthreads();
    const uint32_t mine = tid < kDigits ? seen[0][tid] : 0, all = tid < kDigits ? mine + seen[1][tid] : 0;
    const uint32_t before = before_among_digits(all, of_waves);
    if (tid < kDigits) {
        // One pass sorts all, and its digits are the rows: their counts are the offsets.
        if (a.offsets && a.passes == 1 && blockIdx.x == 0 && (uint32_t)tid <= a.rows) a.offsets[tid] = before;
        uint32_t sum = before + mine;
#pragma unroll
        for (int w = 0; w < kManyWaves; ++w) {
            const uint32_t c = next[w][tid];
            next[w][tid] = sum;
            sum += c;
        }
    }
    __syncthreads();
    auto place = [&](uint32_t at, uint32_t key, uint32_t p) {
        if (s.keys_out) s.keys_out[at] = key;
        if (s.at_out) s.at_out[at] = (int32_t)p;
        else put(a, at, p, key);
    };
    if constexpr (ONCE) {
        if (from + (uint32_t)lane < to) {
            const uint32_t at = next[wave][(key0 >> s.shift) & (kDigits - 1)] + below;
            if constexpr (TALLY) atomicAdd(&tally[at / kManyThreads * kDigits + ((key0 >> (s.shift + kDigitBits)) & (kDigits - 1))], 1u);
            place(at, key0, p0);
        }
        if constexpr (TALLY) {
            __syncthreads();
            uint32_t* counts = s.counts + (uint64_t)s.tiles * kDigits;
            for (uint32_t i = (uint32_t)tid; i < s.tiles * kDigits; i += kManyThreads)
                if (tally[i]) atomicAdd(&counts[i], tally[i]);
        }
        return;
    }
    for (uint32_t base = from; base < to; base += kWave) {
        const uint32_t i = base + (uint32_t)lane;
        const bool there = i < to;
        const uint32_t key = key_at(i), digit = (key >> s.shift) & (kDigits - 1), p = position_at(i);
        same = same_digit(digit, there), below = lanes_below(same);
        uint32_t at = 0;
        if (there) at = next[wave][digit] + below;
        among_lanes();
        if (there && below == 0) next[wave][digit] = at + (uint32_t)__popcll(same);
        among_lanes();
        if (there) place(at, key, p);
    }
}

// offsets where the sorted keys are in memory: a workgroup finds where its rows begin and end, all lanes of a wavefront looking at once, and each of its rows
// looks between.
constexpr int kOffsetThreads = 256;
constexpr uint32_t kKeysMost = 4096;
__device__ __forceinline__ uint32_t first_of_wave(const uint32_t* keys, uint32_t n, uint32_t row) {
    const uint32_t lane = threadIdx.x % kWave;
    uint32_t lo = 0, hi = n;  // it is one of lo .. hi
    while (lo < hi) {
        const uint32_t step = (hi - lo + kWave - 1) / kWave, i = lo + lane * step;
        const uint32_t below = (uint32_t)__popcll(__ballot(i < hi && keys[i < hi ? i : lo] < row));  // of the lanes' keys, sorted as they are
        if (below == 0) return lo;
        hi = min(hi, lo + below * step);
        lo += (below - 1) * step + 1;
    }
    return lo;
}
__global__ __launch_bounds__(kOffsetThreads) void apm_sort_offsets_kernel(const uint32_t* keys, uint32_t n, uint32_t rows, int64_t* offsets) {
    __shared__ uint32_t ends[2];
    __shared__ uint32_t near[kKeysMost];
    const uint32_t first = blockIdx.x * kOffsetThreads, wave = threadIdx.x / kWave;
    if (wave < 2) {
        const uint32_t at = first_of_wave(keys, n, wave == 0 ? first : (uint32_t)min((uint64_t)first + kOffsetThreads, (uint64_t)rows + 1));
        if (threadIdx.x % kWave == 0) ends[wave] = at;
    }
    __syncthreads();
    const uint32_t lo = ends[0], count = ends[1] - lo, r = first + threadIdx.x;
    if (count <= kKeysMost) {
        for (uint32_t i = threadIdx.x; i < count; i += kOffsetThreads) near[i] = keys[lo + i];
        __syncthreads();
        if (r <= rows) offsets[r] = lo + first_of(near, count, r);
    } else if (r <= rows) {
        offsets[r] = lo + first_of(keys + lo, count, r);
    }
}

constexpr int64_t kTilesMost = 512, kTileLeast = kManyThreads;
constexpr uint32_t kOneRows = 4096;        // offsets of so many rows are written by the one workgroup

struct SortShape {
    bool one, tallied;
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
    s.tallied = s.tile == kManyThreads && s.tiles <= kTallied;
    return s;
}
size_t counts_of(const SortShape& s) { return (size_t)(s.tallied ? s.passes : 1) * s.tiles * kDigits; }
size_t to_16(size_t bytes) { return (bytes + 15) / 16 * 16; }
size_t room_of(int64_t n, int64_t rows) {
    const SortShape s = sort_shape(n, rows);
    const size_t words = to_16((size_t)n * 4);
    if (s.one) return words;
    return counts_of(s) * 4 + 4 * words;  // keys and positions, of two passes
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
        else if (a.n <= 2 * kOneThreads) start(apm_sort_one_kernel<2>);
        else start(apm_sort_one_kernel<kOneMost>);
        APM_HIP(hipGetLastError());
    } else {
        char* room = (char*)workspace;
        const size_t words = to_16((size_t)o.n * 4);
        uint32_t* counts = (uint32_t*)room;
        room += counts_of(shape) * 4;
        uint32_t* keys[2] = {(uint32_t*)room, (uint32_t*)(room + words)};
        int32_t* at[2] = {(int32_t*)(room + 2 * words), (int32_t*)(room + 3 * words)};
        for (uint32_t pass = 0; pass < shape.passes; ++pass) {
            const bool last = pass + 1 == shape.passes;
            PassArgs s{};
            s.keys = pass > 0 ? keys[(pass - 1) % 2] : nullptr, s.at = pass > 0 ? at[(pass - 1) % 2] : nullptr;
            s.keys_out = !last || (o.offsets && pass > 0) ? keys[pass % 2] : nullptr, s.at_out = last ? nullptr : at[pass % 2];
            s.counts = counts, s.shift = pass * kDigitBits, s.tile = shape.tile, s.tiles = shape.tiles;
            if (shape.tallied) s.counts += (size_t)pass * shape.tiles * kDigits, s.behind = shape.passes - 1;
            if (pass == 0 || !shape.tallied) hipLaunchKernelGGL(apm_sort_count_kernel, dim3(shape.tiles), dim3(kManyThreads), 0, st, a, s);
            auto start = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(shape.tiles), dim3(kManyThreads), 0, st, a, s); };
            if (shape.tile > kManyThreads) start(apm_sort_place_kernel<false, false>);
            else shape.tallied && !last ? start(apm_sort_place_kernel<true, true>) : start(apm_sort_place_kernel<true, false>);
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

thread_local int64_t t_launch_workgroups = 0;

}  // namespace

int64_t workgroups_of_launch(int threads) { return t_launch_workgroups > 0 ? t_launch_workgroups : max_workgroups(threads) / 2; }

}  // namespace apm

extern "C" int apm_test_set_launch_workgroups(int64_t workgroups) {
    if (workgroups < 0) return apm::fail(APM_EINVAL, "bad argument");
    apm::t_launch_workgroups = workgroups;
    return APM_OK;
}

extern "C" size_t apm_sort_tokens_workspace_bytes(const apm_token_order* o) {
    return !o || apm::check_order(*o) != APM_OK ? 0 : apm::room_of(o->n, o->rows);
}

extern "C" int apm_sort_tokens(const apm_token_order* o, void* workspace, size_t workspace_bytes, void* stream) {
    return apm::guarded([&]() -> int { return apm::sort_tokens(o, workspace, workspace_bytes, stream); });
}
