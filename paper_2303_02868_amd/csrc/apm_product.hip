// Products of tokens with their group's weights: y[t, o] = sum over k of x[t, k] w_g[o, k] + bias_g[o], or with w_g transposed.  bf16 on the matrix cores, sums fp32.
//
// Groups have any number of tokens, which only the device knows.  The grid has room for the most tiles that so many tokens and groups can make; each workgroup
// counts the groups' tiles of rows and finds its own, those behind the last tile leave at once.  Tiles of x and w go into LDS by a ring of stages, each a stretch
// of k, as they lie in memory: k runs along the rows of x, and of w unless that is transposed, which is then read with the transposing loads.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "apm_tok.h"

namespace apm {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) char lds_char;

constexpr int kWave = 64;
constexpr int kFrag = 32, kStep = 16;  // a matrix instruction's tile, and the stretch of k that it takes

// A workgroup's tile of y: WM x WN wavefronts of FM x FN fragments, K of k in a stage, of which there is room in LDS for SLOTS / 2: for a half more where SLOTS is odd,
// which then is x's.
template <int WM_, int WN_, int FM_, int FN_, int K_, int SLOTS_>
struct Tile {
    static constexpr int WM = WM_, WN = WN_, FM = FM_, FN = FN_, K = K_, kSlots = SLOTS_, kStages = SLOTS_ / 2;
    static constexpr bool kHalf = SLOTS_ % 2 != 0;
    static constexpr int kM = WM * FM * kFrag, kN = WN * FN * kFrag, kWaves = WM * WN, kThreads = kWaves * kWave;
    static constexpr int kBytesA = kM * K * 2, kBytesB = kN * K * 2, kStage = kBytesA + kBytesB;
    static constexpr int kA = kBytesA / 1024 / kWaves, kB = kBytesB / 1024 / kWaves;  // 16 bytes a lane, of x and of w, in a stage
    static constexpr int kLds = kStages * kStage + (kHalf ? kBytesA : 0);
    static_assert(!kHalf || kBytesA == kBytesB, "a slot is for either");
    // Where stage j's tile of x or w lies: the slots are taken in turn, x, w, x, w.
    static __device__ __forceinline__ int place_of(int j, bool w) {
        return kHalf ? (2 * j + (w ? 1 : 0)) % kSlots * kBytesA : j % kStages * kStage + (w ? kBytesA : 0);
    }
    static_assert(kA * 1024 * kWaves == kBytesA && kB * 1024 * kWaves == kBytesB, "whole vectors for every lane");
};
// 64 of k in a stage are whole cache lines of rows of x and w (16384 x 4096 x 4096 with 32 of k: 478 us, so 447).
// 256 x 256: the least traffic between L2 and LDS, which bounds the others: loads alone take 341 us of 16384 x 4096 x 4096, products and LDS reads alone 387, together 442 to 489 by
// the card, 1.12 to 1.24 PFLOP/s, at a clock of 1.6 to 1.75 GHz that the matrix cores leave (a library product of that size 415 to 432 on the better card, w as rows of k 479 to 496).
// Of the cycles that a CU is busy the matrix cores are for 73 %, LDS for 29 %.  A half stage more in LDS: input gradients of 8 of 64 groups, 8192 x 1024 x 4096, 114 us without it, so 106.
// One workgroup a CU that goes on from tile to tile, with the next one's loads under the stores, was no faster (8 groups, 16384 x 8192 x 2048: 575 and 578 us).
typedef Tile<2, 4, 4, 2, 64, 5> Large;
// 192 x 256, where 256 x 256 would leave CUs without a tile and this one has one for each at most, as the time is that of a tile then: 6000 x 2048 x 2048
// 53 us by 256 x 256, so 46 to 49; 1500 x 8192 x 2048 52 and 45.  Not through registers.
typedef Tile<2, 4, 3, 2, 64, 4> Lower;
// 128 x 256, where more tiles than CUs or groups of few tokens leave 256 rows half empty: 4096 tokens of 64 experts, 1024 to 4096, 107 to 114 us (108 to 120 by 128 x 128, 157 by 256 x 256),
// 4096 tokens in 8 groups, 4096 to 1024, 61 (71, 102).
typedef Tile<2, 4, 2, 2, 64, 6> Low;
// 128 x 128, two of which share a CU: where 256 x 256 would leave CUs without one (2048 x 2048 x 2048: 43 us, so 25).
typedef Tile<2, 2, 2, 2, 64, 4> Small;
// 64 x 64: short ones (512 x 768 x 768: 8.9 us by 128 x 128, so 5.1), and groups of few tokens (512 tokens of 64 experts, 1024 to 4096: 94 and 85 to 104 by the card).
typedef Tile<2, 2, 1, 1, 64, 6> Tiny;
// Large where rows go through registers: stages of half the length, so that what is on its way fits beside the sums.
typedef Tile<2, 4, 4, 2, 32, 4> LargeAny;
typedef Tile<2, 2, 1, 1, 64, 4> TinyAny;

struct ProductArgs {
    const char* x;
    const char* w;
    const int64_t* offsets;
    apm_vector bias;
    char* y;
    int64_t x_stride, w_stride, w_group_stride, y_stride;
    int64_t tokens;
    int32_t out, in, groups, tiles_n;
    int32_t y_type, accumulate;
    int32_t whole_y;  // its rows, of bf16, are stored in whole vectors
};

// Rows of K elements in LDS are exchanged in vectors of eight, so that what 16 lanes read together of as many rows lies in all of the 64 banks: those that share banks,
// every second row (K = 64) or every fourth, take different vectors.
template <int K> __device__ __forceinline__ int exchange(int row) { return K == 32 ? (row >> 2) & 3 : (row >> 1) & 7; }
template <int K> __device__ __forceinline__ int lds_at(int row, int vec) { return row * (K * 2) + ((vec ^ exchange<K>(row)) << 4); }
template <int K> __device__ __forceinline__ bf16x8 read_fragment(const lds_char* tile, int frag, int step, int lane) {
    typedef __attribute__((address_space(3))) const bf16x8* lds_ptr;
    return *(lds_ptr)(tile + lds_at<K>(frag * kFrag + lane % 32, step * 2 + lane / 32));
}
// Rows of N elements for the transposing loads: 64-byte chunks are exchanged, so that the four rows that such a load takes a chunk of lie in different banks.
template <int N> __device__ __forceinline__ int exchange_t(int row) { return N >= 128 ? row & 3 : N == 64 ? (row >> 1) & 1 : 0; }
template <int N> __device__ __forceinline__ int lds_at_t(int row, int vec) { return row * (N * 2) + (((vec >> 2) ^ exchange_t<N>(row)) << 6) + ((vec & 3) << 4); }
template <int N> __device__ __forceinline__ bf16x8 read_fragment_t(const lds_char* tile, int frag, int step, int lane) {
    typedef __attribute__((address_space(3))) s16x4* lds_ptr;
    const int row = step * kStep + 8 * (lane / 32) + (lane % 16) / 4;
    const lds_char* p = tile + row * (N * 2) + ((frag ^ exchange_t<N>(row)) << 6) + ((lane / 16) & 1) * 32 + (lane & 3) * 8;
    union {
        s16x4 h[2];
        bf16x8 v;
    } u;
    u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)p);
    u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p + 4 * (N * 2)));
    return u.v;
}

__device__ __forceinline__ void group_of(const ProductArgs& a, int g, int64_t* begin, int64_t* end) {
    *begin = 0, *end = a.tokens;
    if (!a.offsets) return;
    *begin = min(max(a.offsets[g], (int64_t)0), a.tokens);
    *end = min(max(a.offsets[g + 1], *begin), a.tokens);
}
// Tiles of rows of groups g .. g + n - 1, M rows each.
template <int M> __device__ __forceinline__ uint32_t row_tiles(const ProductArgs& a, int g, int n) {
    uint32_t t = 0;
#pragma unroll 4
    for (const int end = min(g + n, a.groups); g < end; ++g) {
        int64_t first, last;
        group_of(a, g, &first, &last);
        t += (uint32_t)((last - first + M - 1) / M);
    }
    return t;
}
template <int DPP, int ROWS> __device__ __forceinline__ uint32_t add_from(uint32_t v) {
    return v + (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, DPP, ROWS, 0xf, false);
}
__device__ __forceinline__ uint32_t sum_up_to(uint32_t v) {  // of the lanes up to this one
    v = add_from<0x111, 0xf>(v);  // from 1, 2, 4 and 8 lanes below in a row of 16
    v = add_from<0x112, 0xf>(v);
    v = add_from<0x114, 0xf>(v);
    v = add_from<0x118, 0xf>(v);
    v = add_from<0x142, 0xa>(v);  // a row's last lane to the second and fourth row
    return add_from<0x143, 0xc>(v);  // lane 31 to the upper half
}
__device__ __forceinline__ int64_t of_lane(int64_t v, int lane) {
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, lane));
}

// 16 bytes a lane from memory into LDS, to 16 lane bytes behind `to` (M0); zeros for what lies behind the buffer's end.  In assembly, which does not tell the
// compiler that it writes LDS: told so, it waits for these loads in front of transposing reads of other places (16384 x 4096 x 4096: 500 us).  wait_loads and meet wait.
// ONCE: of what no other workgroup reads, which L2 need not keep.
template <bool ONCE = false> __device__ __forceinline__ void load_to_lds(u32x4 buffer, uint32_t at, uint32_t to) {
    if constexpr (ONCE) asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen nt lds" ::"s"(to), "v"(at), "s"(buffer) : "m0");
    else asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(at), "s"(buffer) : "m0");
}
template <int N> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
// The wavefront's accesses to LDS are done, and so are everyone's.
__device__ __forceinline__ void meet() {
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ u32x4 buffer_of(const char* p, uint32_t bytes) {
    const uint64_t at = (uint64_t)p;
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)at), hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(at >> 32));
    return u32x4{lo, hi & 0xffffu, (uint32_t)__builtin_amdgcn_readfirstlane((int)bytes), 0x00027000u};
}
constexpr uint32_t kNowhere = 0x80000000u;  // behind the end of any buffer here, which product_shape sees to, and so is what is less than 2^30 further on

// The order that the scheduler is to keep in a step: in front of each product its part of the LDS reads for the next step, behind it its part of the loads.
template <int PRODUCTS, int READS, int LOADS, int I = 0> __device__ __forceinline__ void in_turn() {
    if constexpr (I < PRODUCTS) {
        constexpr int kFirst = LOADS > 0 ? 1 : (PRODUCTS + 1) / 2;  // in front of so many products
        if constexpr (I < kFirst) __builtin_amdgcn_sched_group_barrier(0x100, (I + 1) * READS / kFirst - I * READS / kFirst, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x020, (I + 1) * LOADS / PRODUCTS - I * LOADS / PRODUCTS, 0);
        in_turn<PRODUCTS, READS, LOADS, I + 1>();
    }
}

// Which tile a workgroup has.  Workgroups go to the XCDs in turn; each XCD takes a stretch of the order, in which tiles come strip by strip.
// Eight rows of tiles at a time: most of a group's, whose weights then are met once (8 groups, 16384 x 8192 x 2048: 563 us with strips of four, 549 of eight, 565 of sixteen).
constexpr int kXcds = 8, kStrip = 8;
struct Place {
    int64_t row, end;  // the tile's first, and where its group ends
    int group, n_tile;
    bool once;  // the group has no other rows of tiles
    // false: there are fewer tiles.  M: rows of a tile.
    template <int M> __device__ __forceinline__ bool find(const ProductArgs& a, int lane) {
        // Each lane counts the tiles of a stretch of groups; then the lanes look through the stretch that has the tile.
        const int each = (a.groups + kWave - 1) / kWave;
        uint32_t up = 0, rows = (uint32_t)((a.tokens + M - 1) / M);
        int64_t begin = 0;
        end = a.tokens;
        auto count = [&](int g) {  // of one group, or none, which the lane then has in begin and end
            begin = end = 0;
            if (g < a.groups) group_of(a, g, &begin, &end);
            return sum_up_to((uint32_t)((end - begin + M - 1) / M));
        };
        if (a.offsets) {
            up = each == 1 ? count(lane) : sum_up_to(row_tiles<M>(a, lane * each, each));
            rows = (uint32_t)__builtin_amdgcn_readlane((int)up, kWave - 1);
        }
        const uint32_t tiles = rows * (uint32_t)a.tiles_n, nth = blockIdx.x;
        if (nth >= tiles) return false;
        const uint32_t xcd = nth % kXcds, id = xcd * (tiles / kXcds) + min(xcd, tiles % kXcds) + nth / kXcds;
        const uint32_t strip = id / (uint32_t)(kStrip * a.tiles_n), in_strip = id - strip * (uint32_t)(kStrip * a.tiles_n), high = min((uint32_t)kStrip, rows - strip * kStrip);
        uint32_t row_tile = strip * kStrip + in_strip % high;
        n_tile = (int)(in_strip / high);
        group = 0;
        if (a.offsets) {
            int l = 0;
            auto step = [&](int from, int per) {  // lane l has groups from + l per ..; true: the tile is among them
                const uint64_t further = __ballot(up > row_tile);
                if (!further) return false;
                l = __builtin_ctzll(further);
                row_tile -= l > 0 ? (uint32_t)__builtin_amdgcn_readlane((int)up, l - 1) : 0;
                group = from + l * per;
                return true;
            };
            step(0, each);
            if (each > 1) {
                const int from = group, behind = min(from + each, a.groups);
                for (int g = from; g < behind; g += kWave) {
                    up = count(g + lane < behind ? g + lane : a.groups);
                    if (step(g, 1)) break;
                    row_tile -= (uint32_t)__builtin_amdgcn_readlane((int)up, kWave - 1);
                }
            }
            group = __builtin_amdgcn_readfirstlane(group);
            row_tile = (uint32_t)__builtin_amdgcn_readfirstlane((int)row_tile);
            l = __builtin_amdgcn_readfirstlane(l);
            begin = of_lane(begin, l), end = of_lane(end, l);
        }
        row = begin + (int64_t)row_tile * M;
        once = end - begin <= M;
        return row < end;  // groups that overlap can have more tiles than 32 bits count
    }
};

// Eight columns of rows of y from their sums: bias, what y held, rounding.
struct Finish {
    float bias[kVec] = {};
    int col;
    __device__ __forceinline__ Finish(const ProductArgs& a, int group, int col, int n) : col(col) {
        if (!a.bias.data) return;
        const int64_t first = (int64_t)group * a.out + (n > 0 ? col : 0);
        RawAny raw;
        raw.load((const char*)a.bias.data + first * (a.bias.dtype == APM_F32 ? 4 : 2), a.bias.dtype, 0, n);
        raw.get(a.bias.dtype, bias);
    }
    __device__ __forceinline__ void row(const ProductArgs& a, int64_t t, int n, float (&v)[kVec]) const {
        char* to = a.y + t * a.y_stride * (a.y_type == APM_F32 ? 4 : 2);
#pragma unroll
        for (int e = 0; e < kVec; ++e) v[e] += bias[e];
        if (a.accumulate) {
            RawAny old;
            old.load(to, a.y_type, n > 0 ? col : 0, n);
            float f[kVec];
            old.get(a.y_type, f);
#pragma unroll
            for (int e = 0; e < kVec; ++e) v[e] += f[e];
        }
        if (a.y_type == APM_F32) store8<float>(to, col, n, v);
        else if (a.whole_y) store8<bf16, true>(to, col, n, v);
        else store8<bf16>(to, col, n, v);
    }
};

// Eight elements of a row of `width`.  Where fewer of them are there, the row's last eight are loaded, and `fit`, when they are needed, moves those that are down to
// their places and puts zeros in the others: no branch, and no trip to memory for each.
__device__ __forceinline__ u32x4 load_vec(const char* row, int64_t col, int width) {
    if (width < kVec) return width > col ? load_short((const uint16_t*)row + col, width - (int)col) : u32x4{0u, 0u, 0u, 0u};
    return *(const u32x4_any*)(row + min(col, (int64_t)width - kVec) * 2);
}
__device__ __forceinline__ u32x4 fit(u32x4 v, int64_t col, int width) {
    const int n = width - (int)col;
    if (width < kVec || n >= kVec) return v;
    move_down(v, max(n, 1));
    return n > 0 ? v : u32x4{0u, 0u, 0u, 0u};
}

// DIRECT: the tiles go from memory into LDS without passing through registers, which needs whole vectors of sixteen bytes: aligned rows, and widths of a multiple
// of eight.  The other form takes any (2299 tokens in 8 groups, 1664 x 1911: 54 us, 1664 x 1912: 44).
template <class T, bool TRANSPOSED, bool DIRECT>
__global__ __launch_bounds__(T::kThreads) void apm_product_kernel(ProductArgs a) {
    constexpr int FM = T::FM, FN = T::FN, S = T::kStages, kSteps = T::K / kStep;
    static_assert(kSteps % 2 == 0, "two sets of fragments");
    __shared__ __attribute__((aligned(1024))) char lds_all[T::kLds];
    lds_char* const lds = (lds_char*)lds_all;
    const int tid = (int)threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);

    Place at;
    if (!at.find<T::kM>(a, lane)) return;
    const int64_t m0 = at.row, end = at.end;
    const int n0 = at.n_tile * T::kN, group = at.group;
    const char* const w = a.w + (int64_t)group * a.w_group_stride * 2;
    const int stages = (a.in + T::K - 1) / T::K;

    // What a lane brings of a stage, vector by vector.
    constexpr int kVecsK = T::K / kVec, kVecsN = T::kN / kVec;
    uint32_t at_a[T::kA], at_b[T::kB];    // DIRECT: bytes from the tile's corner
    int vec_a[T::kA], vec_b[T::kB];       // the vector's place in k
    u32x4 buf_a, buf_b;
    constexpr int kSets = 2;
    u32x4 ra[kSets][T::kA], rb[kSets][T::kB];  // otherwise: stages on their way
    if constexpr (DIRECT) {
        const int rows_a = (int)min((int64_t)T::kM, end - m0), rows_b = min(T::kN, a.out - n0);
        buf_a = buffer_of(a.x + m0 * a.x_stride * 2, (uint32_t)((rows_a - 1) * a.x_stride * 2 + (int64_t)a.in * 2));
        if constexpr (TRANSPOSED) buf_b = buffer_of(w + (int64_t)n0 * 2, (uint32_t)((a.in - 1) * a.w_stride * 2 + (int64_t)(a.out - n0) * 2));
        else buf_b = buffer_of(w + (int64_t)n0 * a.w_stride * 2, (uint32_t)((rows_b - 1) * a.w_stride * 2 + (int64_t)a.in * 2));
#pragma unroll
        for (int i = 0; i < T::kA; ++i) {
            const int place = (wave * T::kA + i) * kWave + lane, row = place / kVecsK;
            vec_a[i] = (place % kVecsK) ^ exchange<T::K>(row);
            at_a[i] = row < rows_a ? (uint32_t)row * (uint32_t)a.x_stride * 2u + (uint32_t)vec_a[i] * 16u : kNowhere;
        }
#pragma unroll
        for (int i = 0; i < T::kB; ++i) {
            const int place = (wave * T::kB + i) * kWave + lane;
            if constexpr (TRANSPOSED) {
                const int row = place / kVecsN, v = place % kVecsN;
                const int from = ((v >> 2) ^ exchange_t<T::kN>(row)) * 4 + (v & 3);
                at_b[i] = (uint32_t)row * (uint32_t)a.w_stride * 2u + (uint32_t)from * 16u;
                vec_b[i] = row;
            } else {
                const int row = place / kVecsK;
                vec_b[i] = (place % kVecsK) ^ exchange<T::K>(row);
                at_b[i] = row < rows_b ? (uint32_t)row * (uint32_t)a.w_stride * 2u + (uint32_t)vec_b[i] * 16u : kNowhere;
            }
        }
    }
    const uint32_t lds_base = (uint32_t)(uintptr_t)lds;
    // Where a group's weights are read once, groups begin at different k: they would all read the same columns of rows at a time, as a group's own tiles still do, which lie in few of the memory's channels
    // (8000 tokens of 64 experts, 4096 to 1024: 167 us, so 153).
    const int first = !TRANSPOSED && at.once && a.in % T::K == 0 ? (int)((uint32_t)group % (uint32_t)stages) : 0;
    auto stage_at = [&](int j, auto once) { return !once ? j : j + first < stages ? j + first : j + first - stages; };
    // DIRECT: stage j of x, and of w; `whole` if k does not end in it
    auto bring_a = [&](int j, auto whole, auto once) {
        const uint32_t to = lds_base + (uint32_t)T::place_of(j, false) + (uint32_t)wave * (T::kA * 1024u);
        const int k0 = stage_at(j, once) * T::K;
#pragma unroll
        for (int i = 0; i < T::kA; ++i) {
            uint32_t at = at_a[i] + (uint32_t)k0 * 2u;
            if (!whole && k0 + vec_a[i] * kVec >= a.in) at = kNowhere;
            load_to_lds(buf_a, at, to + i * 1024u);
        }
    };
    auto bring_b = [&](int j, auto whole, auto once) {
        const uint32_t to = lds_base + (uint32_t)T::place_of(j, true) + (uint32_t)wave * (T::kB * 1024u);
        const int k0 = stage_at(j, once) * T::K;
#pragma unroll
        for (int i = 0; i < T::kB; ++i) {
            uint32_t at = at_b[i] + (uint32_t)k0 * (TRANSPOSED ? (uint32_t)a.w_stride : 1u) * 2u;
            if (!whole && k0 + (TRANSPOSED ? vec_b[i] : vec_b[i] * kVec) >= a.in) at = kNowhere;
            load_to_lds<decltype(once)::value>(buf_b, at, to + i * 1024u);
        }
    };
    // Rows behind the group's last and columns behind the matrix's are some other ones: what comes of them is not stored.  Behind the end of k
    // there are zeros, in both operands.
    auto fetch = [&](int j, int set) {
        const int k0 = j * T::K;
#pragma unroll
        for (int i = 0; i < T::kA; ++i) {
            const int place = i * T::kThreads + tid;
            ra[set][i] = load_vec(a.x + min(m0 + place / kVecsK, end - 1) * a.x_stride * 2, k0 + place % kVecsK * kVec, a.in);
        }
#pragma unroll
        for (int i = 0; i < T::kB; ++i) {
            const int place = i * T::kThreads + tid;
            if constexpr (TRANSPOSED) rb[set][i] = load_vec(w + (int64_t)min(k0 + place / kVecsN, a.in - 1) * a.w_stride * 2, n0 + place % kVecsN * kVec, a.out);
            else rb[set][i] = load_vec(w + (int64_t)min(n0 + place / kVecsK, a.out - 1) * a.w_stride * 2, k0 + place % kVecsK * kVec, a.in);
        }
    };
    const bool n_ends = TRANSPOSED && n0 + T::kN > a.out;
    typedef __attribute__((address_space(3))) u32x4* lds_vec;
    auto put_as = [&](int j, int set, auto ends) {
        lds_char *const to_a = lds + T::place_of(j, false), *const to_b = lds + T::place_of(j, true);
        const int k0 = j * T::K;
#pragma unroll
        for (int i = 0; i < T::kA; ++i) {
            const int place = i * T::kThreads + tid;
            u32x4 v = ra[set][i];
            if (ends) v = fit(v, k0 + place % kVecsK * kVec, a.in);
            *(lds_vec)(to_a + lds_at<T::K>(place / kVecsK, place % kVecsK)) = v;
        }
#pragma unroll
        for (int i = 0; i < T::kB; ++i) {
            const int place = i * T::kThreads + tid;
            u32x4 v = rb[set][i];
            if constexpr (TRANSPOSED) {
                if (ends) v = k0 + place / kVecsN < a.in ? fit(v, n0 + place % kVecsN * kVec, a.out) : u32x4{0u, 0u, 0u, 0u};
                *(lds_vec)(to_b + lds_at_t<T::kN>(place / kVecsN, place % kVecsN)) = v;
            } else {
                if (ends) v = fit(v, k0 + place % kVecsK * kVec, a.in);
                *(lds_vec)(to_b + lds_at<T::K>(place / kVecsK, place % kVecsK)) = v;
            }
        }
    };
    auto put = [&](int j, int set) {
        if (n_ends || j * T::K + T::K > a.in) put_as(j, set, std::true_type());
        else put_as(j, set, std::false_type());
    };

    f32x16 acc[FM][FN];
#pragma unroll
    for (int m = 0; m < FM; ++m)
#pragma unroll
        for (int n = 0; n < FN; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[m][n][r] = 0.0f;
    const int wm = wave / T::WN * FM, wn = wave % T::WN * FN;  // the wavefront's first fragments
    bf16x8 fa[2][FM], fb[2][FN];
    auto read = [&](int j, int step) {
        const lds_char *const from_a = lds + T::place_of(j, false), *const from_b = lds + T::place_of(j, true);
#pragma unroll
        for (int n = 0; n < FN; ++n) {
            if constexpr (TRANSPOSED) fb[step % 2][n] = read_fragment_t<T::kN>(from_b, wn + n, step, lane);
            else fb[step % 2][n] = read_fragment<T::K>(from_b, wn + n, step, lane);
        }
#pragma unroll
        for (int m = 0; m < FM; ++m) fa[step % 2][m] = read_fragment<T::K>(from_a, wm + m, step, lane);
    };
    auto multiply = [&](int step) {
#pragma unroll
        for (int m = 0; m < FM; ++m)
#pragma unroll
            for (int n = 0; n < FN; ++n) acc[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[step % 2][m], fb[step % 2][n], acc[m][n], 0, 0, 0);
    };
    constexpr int kReads = FM + (TRANSPOSED ? 2 : 1) * FN, kLoads = T::kA + T::kB;
    constexpr int kExtra = T::kHalf ? T::kA : 0;  // loads of a stage of x that is under way beyond the whole ones
    auto bring = [&](int j, auto whole_a, auto whole_b, auto once) {  // what takes the place of stage j - S: of w stage j, of x that or the next one
        const int ja = T::kHalf ? j + 1 : j;
        if (whole_b || j < stages) bring_b(j, whole_b, once);
        if (whole_a || ja < stages) bring_a(ja, whole_a, once);
    };
    auto is_whole = [&](int j) { return (j + 1) * T::K <= a.in; };
    // Fragments are read a step ahead.  Before a stage's last step everybody has read that stage, whose place is filled anew, and the next stage is there.
    auto others = [&](int j) {  // all steps of stage j but the last
#pragma unroll
        for (int s = 0; s + 1 < kSteps; ++s) {
            read(j, s + 1);
            multiply(s);
            in_turn<FM * FN, kReads, 0>();
        }
    };
    auto turn = [&](int j, auto&& fill) {
        meet();
        read(j + 1, 0);
        fill();
        multiply(kSteps - 1);
        in_turn<FM * FN, kReads, DIRECT ? kLoads : 0>();
        others(j + 1);
    };
    if constexpr (DIRECT) {
        auto all = [&](auto once) {
            if (T::kHalf) bring_a(0, is_whole(0), once);
#pragma unroll
            for (int j = 0; j < S; ++j) bring(j, is_whole(T::kHalf ? j + 1 : j), is_whole(j), once);
            if (S + (T::kHalf ? 1 : 0) <= stages) wait_loads<(S - 1) * kLoads + kExtra>();
            else wait_loads<0>();
            meet();
            read(0, 0);
            others(0);
            int j = 0;
            for (const int whole = a.in / T::K - (T::kHalf ? 1 : 0); j + S < whole; ++j) {
                wait_loads<(S - 2) * kLoads + kExtra>();
                turn(j, [&] { bring(j + S, std::true_type(), std::true_type(), once); });
            }
            for (; j + 1 < stages; ++j) {
                if (j + S + (T::kHalf ? 1 : 0) <= stages) wait_loads<(S - 2) * kLoads + kExtra>();
                else wait_loads<0>();
                turn(j, [&] { bring(j + S, is_whole(T::kHalf ? j + S + 1 : j + S), is_whole(j + S), once); });
            }
        };
        // Weights that one row of tiles reads, non-temporally: 4096 and 512 tokens in 64 groups, 4096 x 1024, 130 and 103 us, 137 and 111 without (weights that come more
        // often are better kept: 16384 x 4096 x 4096 would take 474 instead of 456).  So is y stored where a
        // wavefront's instruction fills whole lines (126 and 103, 448; fp32 rows of 4095 by halves of vectors: 183 us, so 163).
        if (at.once) all(std::true_type());
        else all(std::false_type());
    } else {
#pragma unroll
        for (int j = 0; j < kSets; ++j)
            if (j < stages) fetch(j, j);
#pragma unroll
        for (int j = 0; j < kSets; ++j)
            if (j < stages) put(j, j);
#pragma unroll
        for (int j = kSets; j < 2 * kSets; ++j)
            if (j < stages) fetch(j, j % kSets);
        meet();
        read(0, 0);
        others(0);
        static_assert(S == kSets, "a stage's set of registers goes where the stage two before it was");
        for (int j = 0; j + 1 < stages; j += kSets) {
#pragma unroll
            for (int u = 0; u < kSets; ++u) {
                if (j + u + 1 >= stages) break;
                turn(j + u, [&] {
                    if (j + u + S < stages) put(j + u + S, u);
                    if (j + u + S + kSets < stages) fetch(j + u + S + kSets, u);
                });
            }
        }
    }
    multiply(kSteps - 1);
    meet();

    // Lane l has column l mod 32 of a fragment's tile, rows 8 (r / 4) + 4 (l / 32) + r mod 4 in register r.  Rows are stored in whole vectors: half a fragment's
    // rows at a time go through LDS, each wavefront for itself.
    constexpr int kRow = FN * kFrag + 4, kPer = FN * kFrag / kVec, kRowsAtOnce = kWave / kPer;
    static_assert(T::kWaves * 16 * kRow * 4 <= T::kLds, "the wavefronts' rows fit");
    typedef __attribute__((address_space(3))) float lds_float;
    lds_float* const mine = (lds_float*)lds + wave * 16 * kRow;
    const int c = lane % kPer * kVec, col = n0 + wn * kFrag + c, there = max(0, min(kVec, a.out - col));
    const Finish finish(a, group, col, there);
#pragma unroll
    for (int m = 0; m < FM; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h) {  // registers 8 h .. 8 h + 7: rows 16 h .. 16 h + 15
            among_lanes();
#pragma unroll
            for (int r = 0; r < 8; ++r)
#pragma unroll
                for (int n = 0; n < FN; ++n) mine[(8 * (r / 4) + 4 * (lane / 32) + r % 4) * kRow + n * kFrag + lane % 32] = acc[m][n][8 * h + r];
            among_lanes();
#pragma unroll
            for (int i = 0; i < 16 / kRowsAtOnce; ++i) {
                const int row = i * kRowsAtOnce + lane / kPer;
                const int64_t t = m0 + (wm + m) * kFrag + 16 * h + row;
                float v[kVec];
#pragma unroll
                for (int e = 0; e < kVec; ++e) v[e] = mine[row * kRow + c + e];
                finish.row(a, t, t < end ? there : 0, v);
            }
        }
}

// Few rows: HBM-bound by the weights, and too few tiles for the chip unless they are small.  Each of a workgroup's wavefronts takes every fourth stage of k of the
// same 32 x 32 tile, by a ring in LDS of its own, so that nobody waits for anybody until the four sums come together at the end.  Two tokens of two of 64 groups,
// 4096 x 1024: 4.5 us a call among others, 6.2 by itself (8.6 among others by 64 x 64), one token, 768 x 768: 3.7 (4.9), 56 tokens of 8 groups, 1152 x 3776: 11 (18).
template <int FM_, int FN_, int STAGES_>
struct Few {
    static constexpr int FM = FM_, FN = FN_, kStages = STAGES_, K = 64, kWaves = 4, kThreads = kWaves * kWave;
    static constexpr int kM = FM * kFrag, kN = FN * kFrag, kBytesA = kM * K * 2, kBytesB = kN * K * 2, kStage = kBytesA + kBytesB;
    static constexpr int kA = kBytesA / 1024, kB = kBytesB / 1024;
};
typedef Few<1, 1, 4> Strips;
// 64 x 64, for few tiles and long sums: 64 tokens, 2048 to 8192: 10.5 us (15.7 by four wavefronts that share the stages, 11.7 by 32 x 32), 512 tokens, 4096 to 1024: 16.0 (18.7, 16.3).
// Not through registers.
typedef Few<2, 2, 2> Squares;

template <class T, bool TRANSPOSED, bool DIRECT>
__global__ __launch_bounds__(T::kThreads) void apm_product_few_kernel(ProductArgs a) {
    constexpr int FM = T::FM, FN = T::FN, S = T::kStages, kSteps = T::K / kStep, kRow = T::kN + 4;
    constexpr int kRing = (DIRECT ? S : 1) * T::kStage, kSums = T::kM * kRow * 4;
    __shared__ __attribute__((aligned(1024))) char lds_all[T::kWaves * (kRing > kSums ? kRing : kSums)];
    lds_char* const lds = (lds_char*)lds_all;
    const int tid = (int)threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    Place place;
    if (!place.find<T::kM>(a, lane)) return;
    const int64_t m0 = place.row, end = place.end;
    const int n0 = place.n_tile * T::kN;
    const char* const w = a.w + (int64_t)place.group * a.w_group_stride * 2;
    lds_char* const ring = lds + wave * kRing;
    const uint32_t ring_at = (uint32_t)(uintptr_t)ring;
    const int stages = (a.in + T::K - 1) / T::K, mine = (stages - wave + T::kWaves - 1) / T::kWaves;  // the wavefront's: wave, wave + 4, ..
    constexpr int kVecsK = T::K / kVec, kVecsN = T::kN / kVec;

    uint32_t at_a[T::kA], at_b[T::kB];
    int vec_a[T::kA], vec_b[T::kB];
    constexpr int kSets = 2;
    u32x4 buf_a, buf_b, ra[kSets][T::kA], rb[kSets][T::kB];
    if constexpr (DIRECT) {
        const int rows_a = (int)min((int64_t)T::kM, end - m0), rows_b = min(T::kN, a.out - n0);
        buf_a = buffer_of(a.x + m0 * a.x_stride * 2, (uint32_t)((rows_a - 1) * a.x_stride * 2 + (int64_t)a.in * 2));
        if constexpr (TRANSPOSED) buf_b = buffer_of(w + (int64_t)n0 * 2, (uint32_t)((a.in - 1) * a.w_stride * 2 + (int64_t)(a.out - n0) * 2));
        else buf_b = buffer_of(w + (int64_t)n0 * a.w_stride * 2, (uint32_t)((rows_b - 1) * a.w_stride * 2 + (int64_t)a.in * 2));
#pragma unroll
        for (int i = 0; i < T::kA; ++i) {
            const int at = i * kWave + lane, row = at / kVecsK;
            vec_a[i] = ((at % kVecsK) ^ exchange<T::K>(row)) * kVec;
            at_a[i] = row < rows_a ? (uint32_t)row * (uint32_t)a.x_stride * 2u + (uint32_t)vec_a[i] * 2u : kNowhere;
        }
#pragma unroll
        for (int i = 0; i < T::kB; ++i) {
            const int at = i * kWave + lane;
            if constexpr (TRANSPOSED) {
                const int row = at / kVecsN, v = at % kVecsN;
                vec_b[i] = row;
                at_b[i] = (uint32_t)row * (uint32_t)a.w_stride * 2u + (uint32_t)(((v >> 2) ^ exchange_t<T::kN>(row)) * 4 + (v & 3)) * 16u;
            } else {
                const int row = at / kVecsK;
                vec_b[i] = ((at % kVecsK) ^ exchange<T::K>(row)) * kVec;
                at_b[i] = row < rows_b ? (uint32_t)row * (uint32_t)a.w_stride * 2u + (uint32_t)vec_b[i] * 2u : kNowhere;
            }
        }
    }
    auto bring = [&](int i) {  // the wavefront's i-th stage
        const int k0 = (wave + i * T::kWaves) * T::K;
        const uint32_t to = ring_at + (uint32_t)(i % S) * T::kStage;
#pragma unroll
        for (int u = 0; u < T::kA; ++u) load_to_lds(buf_a, k0 + vec_a[u] < a.in ? at_a[u] + (uint32_t)k0 * 2u : kNowhere, to + u * 1024u);
#pragma unroll
        for (int u = 0; u < T::kB; ++u)
            load_to_lds(buf_b, k0 + vec_b[u] < a.in ? at_b[u] + (uint32_t)k0 * (TRANSPOSED ? (uint32_t)a.w_stride : 1u) * 2u : kNowhere, to + T::kBytesA + u * 1024u);
    };
    auto fetch = [&](int j, int set) {
        const int k0 = (wave + j * T::kWaves) * T::K;
#pragma unroll
        for (int i = 0; i < T::kA; ++i) {
            const int at = i * kWave + lane;
            ra[set][i] = load_vec(a.x + min(m0 + at / kVecsK, end - 1) * a.x_stride * 2, k0 + at % kVecsK * kVec, a.in);
        }
#pragma unroll
        for (int i = 0; i < T::kB; ++i) {
            const int at = i * kWave + lane;
            if constexpr (TRANSPOSED) rb[set][i] = load_vec(w + (int64_t)min(k0 + at / kVecsN, a.in - 1) * a.w_stride * 2, n0 + at % kVecsN * kVec, a.out);
            else rb[set][i] = load_vec(w + (int64_t)min(n0 + at / kVecsK, a.out - 1) * a.w_stride * 2, k0 + at % kVecsK * kVec, a.in);
        }
    };
    const bool n_ends = TRANSPOSED && n0 + T::kN > a.out;
    typedef __attribute__((address_space(3))) u32x4* lds_vec;
    auto put_as = [&](int j, int set, auto ends) {
        lds_char *const to_a = ring, *const to_b = ring + T::kBytesA;
        const int k0 = (wave + j * T::kWaves) * T::K;
#pragma unroll
        for (int i = 0; i < T::kA; ++i) {
            const int at = i * kWave + lane;
            u32x4 v = ra[set][i];
            if (ends) v = fit(v, k0 + at % kVecsK * kVec, a.in);
            *(lds_vec)(to_a + lds_at<T::K>(at / kVecsK, at % kVecsK)) = v;
        }
#pragma unroll
        for (int i = 0; i < T::kB; ++i) {
            const int at = i * kWave + lane;
            u32x4 v = rb[set][i];
            if constexpr (TRANSPOSED) {
                if (ends) v = k0 + at / kVecsN < a.in ? fit(v, n0 + at % kVecsN * kVec, a.out) : u32x4{0u, 0u, 0u, 0u};
                *(lds_vec)(to_b + lds_at_t<T::kN>(at / kVecsN, at % kVecsN)) = v;
            } else {
                if (ends) v = fit(v, k0 + at % kVecsK * kVec, a.in);
                *(lds_vec)(to_b + lds_at<T::K>(at / kVecsK, at % kVecsK)) = v;
            }
        }
    };
    auto put = [&](int j, int set) {
        if (n_ends || (wave + j * T::kWaves) * T::K + T::K > a.in) put_as(j, set, std::true_type());
        else put_as(j, set, std::false_type());
    };

    f32x16 acc[FM][FN];
#pragma unroll
    for (int m = 0; m < FM; ++m)
#pragma unroll
        for (int n = 0; n < FN; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[m][n][r] = 0.0f;
    auto multiply = [&](const lds_char* from) {
        bf16x8 fa[kSteps][FM], fb[kSteps][FN];
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
#pragma unroll
            for (int m = 0; m < FM; ++m) fa[s][m] = read_fragment<T::K>(from, m, s, lane);
#pragma unroll
            for (int n = 0; n < FN; ++n) {
                if constexpr (TRANSPOSED) fb[s][n] = read_fragment_t<T::kN>(from + T::kBytesA, n, s, lane);
                else fb[s][n] = read_fragment<T::K>(from + T::kBytesA, n, s, lane);
            }
        }
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
#pragma unroll
            for (int m = 0; m < FM; ++m)
#pragma unroll
                for (int n = 0; n < FN; ++n) acc[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[s][m], fb[s][n], acc[m][n], 0, 0, 0);
    };
    if constexpr (DIRECT) {
        constexpr int kLoads = T::kA + T::kB;
#pragma unroll
        for (int i = 0; i < S; ++i)
            if (i < mine) bring(i);
        for (int i = 0; i < mine; ++i) {
            if (i + S <= mine) wait_loads<(S - 1) * kLoads>();
            else wait_loads<0>();
            multiply(ring + i % S * T::kStage);
            if (i + S < mine) {
                wait_lds();  // the stage's fragments are read
                bring(i + S);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < kSets; ++i)
            if (i < mine) fetch(i, i);
        for (int i = 0; i < mine; i += kSets) {
#pragma unroll
            for (int u = 0; u < kSets; ++u) {
                if (i + u >= mine) break;
                among_lanes();
                put(i + u, u);
                if (i + u + kSets < mine) fetch(i + u + kSets, u);
                among_lanes();
                multiply(ring);
            }
        }
    }
    meet();
    typedef __attribute__((address_space(3))) float lds_float;
    lds_float* const sums = (lds_float*)lds;
    constexpr int kPart = T::kM * kRow;
#pragma unroll
    for (int m = 0; m < FM; ++m)
#pragma unroll
        for (int n = 0; n < FN; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) sums[wave * kPart + (m * kFrag + 8 * (r / 4) + 4 * (lane / 32) + r % 4) * kRow + n * kFrag + lane % 32] = acc[m][n][r];
    __syncthreads();
    constexpr int kPer = T::kN / kVec, kRowsAtOnce = T::kThreads / kPer;
    const int c = tid % kPer * kVec, there = max(0, min(kVec, a.out - (n0 + c)));
    const Finish finish(a, place.group, n0 + c, there);
#pragma unroll
    for (int i = 0; i < (T::kM + kRowsAtOnce - 1) / kRowsAtOnce; ++i) {
        const int row = i * kRowsAtOnce + tid / kPer;
        if (row >= T::kM || m0 + row >= end) continue;
        float v[kVec];
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
            const lds_float* p = sums + row * kRow + c + e;
            v[e] = (p[0] + p[kPart]) + (p[2 * kPart] + p[3 * kPart]);
        }
        finish.row(a, m0 + row, there, v);
    }
}

int check_product(const apm_grouped_product_desc& p) {
    if (p.tokens < 0 || p.tokens > ((int64_t)1 << 40) || p.out < 1 || p.in < 1 || p.out > kMostCols || p.in > kMostCols || p.n_groups < 0 || p.n_groups > APM_MAX_GROUPS)
        return fail(APM_EINVAL, "bad size: %lld tokens, %lld x %lld, %lld groups", (long long)p.tokens, (long long)p.out, (long long)p.in, (long long)p.n_groups);
    if ((p.n_groups > 0) != (p.offsets != nullptr)) return fail(APM_EINVAL, "offsets and n_groups contradict each other");
    if (!aligned_to(p.offsets, 8)) return fail(APM_EINVAL, "offsets are not aligned to their elements");
    const int64_t w_rows = p.transposed ? p.in : p.out, w_cols = p.transposed ? p.out : p.in;
    int rc = check_matrix("x", p.x, p.tokens, p.in, false);
    if (rc == APM_OK && p.tokens > 0 && p.x.dtype != APM_BF16) rc = fail(APM_EINVAL, "x must be bf16");
    if (rc == APM_OK) rc = check_matrix("w", p.w, w_rows, w_cols, false);
    if (rc == APM_OK && p.w.dtype != APM_BF16) rc = fail(APM_EINVAL, "w must be bf16");
    if (rc == APM_OK) rc = check_vector("bias", p.bias);
    if (rc == APM_OK) rc = check_matrix("y", p.y, p.tokens, p.out, true);
    if (rc == APM_OK && p.n_groups > 1 && (p.w_group_stride < 0 || p.w_group_stride > ((int64_t)1 << 56) / p.n_groups)) rc = fail(APM_EINVAL, "w's groups are too far apart");
    return rc;
}

enum { kLarge, kLower, kLow, kSmall, kTiny, kSquares, kFew, kTiles };
struct ProductShape {
    int which;  // kTiles: no tile of which a grid holds enough
    bool direct;
    int64_t tiles_m, tiles_n;
};
// Which tile: estimated in us, from calls that were timed; over 151 drawn sizes and groups the choice is the fastest of the seven or within 15 % or 1.5 us of it, but for
// groups of which few have tokens (2970 tokens in 10 of 64, 768 to 7836: 93 and 73 us) and a short k of odd length (9557 tokens, 79 to 4983: 47 and 36).  There is no term for
// memory, and groups of some 200 tokens with a long k, where it decides, can do better, too (1600 tokens of 8 groups, 4096 to 4096: 106 and 85).  A
// workgroup that has a CU for itself takes `start` and `alone` for each 64 of k; a CU that is full, `busy` for that of each workgroup it has, and `round` more for each.
struct TileCost {
    int rows, cols, threads;
    int per_cu;  // workgroups that start together
    double start, round, alone[2], busy[2];  // through registers, direct
};
constexpr double kNever = 1e30;
constexpr TileCost kCost[kTiles] = {
    {Large::kM, Large::kN, Large::kThreads, 1, 8.0, 6.0, {1.9, 1.08}, {2.5, 1.63}},
    {Lower::kM, Lower::kN, Lower::kThreads, 1, 7.0, 0.0, {kNever, 0.85}, {kNever, 1.24}},
    {Low::kM, Low::kN, Low::kThreads, 1, 7.0, 3.0, {kNever, 0.6}, {kNever, 0.88}},
    {Small::kM, Small::kN, Small::kThreads, 2, 4.6, 1.0, {0.95, 0.39}, {0.8, 0.49}},
    {Tiny::kM, Tiny::kN, Tiny::kThreads, 0, 2.6, 0.35, {0.5, 0.25}, {0.33, 0.185}},
    {Squares::kM, Squares::kN, Squares::kThreads, 1, 5.2, 3.0, {kNever, 0.165}, {kNever, 0.2}},
    {Strips::kM, Strips::kN, Strips::kThreads, 0, 2.7, 2.2, {0.31, 0.085}, {0.13, 0.1}},
};
constexpr double kCus = 256.0;
double cost_of(const apm_grouped_product_desc& p, const TileCost& c, bool direct) {
    // Groups may be empty, but that is not known here: half of the last tile of each is taken for used.
    const double groups = (double)std::min(p.n_groups, p.tokens);
    const double rows = p.n_groups > 1 ? std::max(groups, (double)p.tokens / c.rows + 0.5 * groups) : (double)div_up(p.tokens, c.rows);
    const double load = rows * (double)div_up(p.out, c.cols) / kCus, stages = (double)div_up(p.in, 64);
    if (c.rows == Lower::kM && load > 1.0) return kNever;
    // Workgroups of a CU that is not full get in each other's way less than in proportion.
    const bool part = load <= std::max(1, c.per_cu);
    const double rounds = part || !c.per_cu ? load : std::ceil(load / c.per_cu) * c.per_cu;
    const double crowd = part && c.per_cu > 1 ? 1.2 - 0.25 * std::max(0.0, load - 1.0) : 1.0;
    return c.start + std::max(0.0, rounds - 1.0) * c.round + stages * std::max(c.alone[direct], rounds * c.busy[direct] * crowd);
}
ProductShape product_shape(const apm_grouped_product_desc& p) {
    ProductShape s{};
    const int64_t reach = (int64_t)1 << 30, w_rows = p.transposed ? p.in + 4 * Large::K : Large::kN;
    // Rows that overlap can be wider than they are apart: what a tile's loads go by ends at 2^31 bytes all the same.
    auto ends = [&](int64_t rows, const apm_matrix& m, int64_t cols) { return (rows - 1) * m.stride + cols <= reach; };
    s.direct = aligned_to(p.x.data, 16) && aligned_to(p.w.data, 16) && p.x.stride % kVec == 0 && p.w.stride % kVec == 0 && (p.n_groups < 2 || p.w_group_stride % kVec == 0) &&
               p.in % kVec == 0 && (!p.transposed || p.out % kVec == 0) && p.x.stride < reach / Large::kM && p.w.stride < reach / w_rows && p.in < reach / 4 && p.out < reach / 4 &&
               ends(Large::kM, p.x, p.in) && ends(p.transposed ? p.in : Large::kN, p.w, p.transposed ? p.out : p.in);
    s.which = kTiles;
    double least = kNever;
    for (int i = 0; i < kTiles; ++i) {
        // tokens fill whole tiles but for the last of each group
        const int64_t groups = std::max<int64_t>(1, p.n_groups), m = std::min(p.tokens, p.tokens / kCost[i].rows + std::min(groups, p.tokens)), n = div_up(p.out, kCost[i].cols);
        const double cost = cost_of(p, kCost[i], s.direct);
        if (cost >= least || m > max_workgroups(kCost[i].threads) / n) continue;
        s.which = i, s.tiles_m = m, s.tiles_n = n, least = cost;
    }
    return s;
}

// ANY: the tile through registers, of the same rows and columns, which the grid is counted for; void: there is no such form, and cost_of never takes it.
template <class T, class ANY = T> hipError_t launch_product(const ProductArgs& a, bool transposed, bool direct, unsigned workgroups, hipStream_t s) {
    auto start = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(workgroups), dim3(T::kThreads), 0, s, a); };
    if (direct) {
        transposed ? start(apm_product_kernel<T, true, true>) : start(apm_product_kernel<T, false, true>);
    } else if constexpr (std::is_void<ANY>::value) {
        return hipErrorInvalidValue;
    } else {
        static_assert(ANY::kM == T::kM && ANY::kN == T::kN && ANY::kThreads == T::kThreads, "the same tile of y");
        transposed ? start(apm_product_kernel<ANY, true, false>) : start(apm_product_kernel<ANY, false, false>);
    }
    return hipGetLastError();
}
template <class T, class ANY = T> hipError_t launch_few(const ProductArgs& a, bool transposed, bool direct, unsigned workgroups, hipStream_t s) {
    auto start = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(workgroups), dim3(T::kThreads), 0, s, a); };
    if (direct) {
        transposed ? start(apm_product_few_kernel<T, true, true>) : start(apm_product_few_kernel<T, false, true>);
    } else if constexpr (std::is_void<ANY>::value) {
        return hipErrorInvalidValue;
    } else {
        static_assert(ANY::kM == T::kM && ANY::kN == T::kN && ANY::kThreads == T::kThreads, "the same tile of y");
        transposed ? start(apm_product_few_kernel<ANY, true, false>) : start(apm_product_few_kernel<ANY, false, false>);
    }
    return hipGetLastError();
}

int grouped_product(const apm_grouped_product_desc* pp, void* workspace, size_t workspace_bytes, void* stream) {
    if (!pp) return fail(APM_EINVAL, "missing argument");
    const apm_grouped_product_desc& p = *pp;
    int rc = check_product(p);
    if (rc == APM_OK) rc = check_room(workspace, workspace_bytes, 0);
    if (rc != APM_OK || p.tokens == 0) return rc;
    ProductArgs a{};
    a.x = (const char*)p.x.data, a.w = (const char*)p.w.data, a.offsets = p.offsets, a.bias = p.bias, a.y = (char*)p.y.data;
    a.x_stride = p.x.stride, a.w_stride = p.w.stride, a.w_group_stride = p.n_groups > 1 ? p.w_group_stride : 0, a.y_stride = p.y.stride;
    a.tokens = p.tokens, a.out = (int32_t)p.out, a.in = (int32_t)p.in, a.groups = (int32_t)std::max<int64_t>(1, p.n_groups);
    a.y_type = p.y.dtype, a.accumulate = p.accumulate;
    a.whole_y = p.y.dtype == APM_BF16 && aligned_to(p.y.data, 16) && p.y.stride % kVec == 0;
    const ProductShape s = product_shape(p);
    a.tiles_n = (int32_t)s.tiles_n;
    if (s.which == kTiles) return fail(APM_EINVAL, "y is too large for one product");
    const unsigned n = (unsigned)(s.tiles_m * s.tiles_n);
    const hipStream_t st = (hipStream_t)stream;
    APM_HIP(s.which == kLarge   ? (launch_product<Large, LargeAny>)(a, p.transposed, s.direct, n, st)
            : s.which == kLower ? (launch_product<Lower, void>)(a, p.transposed, s.direct, n, st)
            : s.which == kLow   ? (launch_product<Low, void>)(a, p.transposed, s.direct, n, st)
            : s.which == kSmall ? launch_product<Small>(a, p.transposed, s.direct, n, st)
            : s.which == kTiny  ? (launch_product<Tiny, TinyAny>)(a, p.transposed, s.direct, n, st)
            : s.which == kSquares ? (launch_few<Squares, void>)(a, p.transposed, s.direct, n, st)
                                  : launch_few<Strips>(a, p.transposed, s.direct, n, st));
    return APM_OK;
}

}  // namespace
}  // namespace apm

extern "C" size_t apm_grouped_product_workspace_bytes(const apm_grouped_product_desc*) { return 0; }

extern "C" int apm_grouped_product(const apm_grouped_product_desc* p, void* workspace, size_t workspace_bytes, void* stream) {
    return apm::guarded([&]() -> int { return apm::grouped_product(p, workspace, workspace_bytes, stream); });
}

extern "C" int apm_test_grouped_product_tile(const apm_grouped_product_desc* p) {
    if (!p || apm::check_product(*p) != APM_OK) return 0;
    const apm::ProductShape s = apm::product_shape(*p);
    if (s.which == apm::kTiles) return 0;
    const int rows = apm::kCost[s.which].rows;
    return s.which == apm::kLow || s.which == apm::kSquares ? -rows : rows;
}
