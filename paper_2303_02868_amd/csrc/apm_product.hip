// Products of tokens with their group's weights: y[t, o] = sum over k of x[t, k] w_g[o, k] + bias_g[o], or with w_g transposed.  bf16 on the matrix cores, sums fp32.
//
// Groups have any number of tokens, which only the device knows.  The grid has room for the most tiles that so many tokens and groups can make; each workgroup
// counts the groups' tiles of rows and finds its own, those behind the last tile leave at once.  Tiles of x and w go into LDS by a ring of stages, each a stretch
// of k, as they lie in memory: k runs along the rows of x, and of w unless that is transposed, which is then read with the transposing loads.
#include <algorithm>

#include "apm_tok.h"

namespace apm {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) char lds_char;

constexpr int kWave = 64;
constexpr int kFrag = 32, kStep = 16;  // a matrix instruction's tile, and the stretch of k that it takes

// A workgroup's tile of y: WM x WN wavefronts of FM x FN fragments, K of k in a stage, STAGES of them in LDS.
template <int WM_, int WN_, int FM_, int FN_, int K_, int STAGES_>
struct Tile {
    static constexpr int WM = WM_, WN = WN_, FM = FM_, FN = FN_, K = K_, kStages = STAGES_;
    static constexpr int kM = WM * FM * kFrag, kN = WN * FN * kFrag, kWaves = WM * WN, kThreads = kWaves * kWave;
    static constexpr int kBytesA = kM * K * 2, kBytesB = kN * K * 2, kStage = kBytesA + kBytesB;
    static constexpr int kA = kBytesA / 1024 / kWaves, kB = kBytesB / 1024 / kWaves;  // 16 bytes a lane, of x and of w, in a stage
    static_assert(kA * 1024 * kWaves == kBytesA && kB * 1024 * kWaves == kBytesB, "whole vectors for every lane");
};
typedef Tile<2, 4, 4, 2, 32, 4> Large;
typedef Tile<2, 2, 2, 2, 32, 4> Small;
typedef Tile<2, 2, 1, 1, 64, 3> Tiny;
typedef Tile<1, 4, 1, 1, 64, 4> Thin;

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
};

// Rows of K elements in LDS are exchanged in vectors of eight, so that those of eight neighbouring rows that a fragment is read from lie in different banks.
template <int K> __device__ __forceinline__ int exchange(int row) { return K == 32 ? (row >> 1) & 3 : row & 7; }
template <int K> __device__ __forceinline__ int lds_at(int row, int vec) { return row * (K * 2) + ((vec ^ exchange<K>(row)) << 4); }
template <int K> __device__ __forceinline__ bf16x8 read_fragment(const lds_char* tile, int frag, int step, int lane) {
    typedef __attribute__((address_space(3))) const bf16x8* lds_ptr;
    return *(lds_ptr)(tile + lds_at<K>(frag * kFrag + lane % 32, step * 2 + lane / 32));
}
// Rows of N elements for the transposing loads: 64-byte chunks are exchanged, so that the four rows that such a load takes a chunk of lie in different banks.
template <int N> __device__ __forceinline__ int exchange_t(int row) { return N >= 128 ? row & 3 : (row >> 1) & 1; }
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
// The tiles of rows of 64 groups from g0 on: lane l gets how many there are in front of group g0 + l + 1.
template <int M> __device__ __forceinline__ uint32_t tiles_up_to(const ProductArgs& a, int g0, int lane) {
    uint32_t t = 0;
    if (g0 + lane < a.groups) {
        int64_t begin, end;
        group_of(a, g0 + lane, &begin, &end);
        t = (uint32_t)((end - begin + M - 1) / M);
    }
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
        const uint32_t o = __shfl_up(t, d);
        if (lane >= d) t += o;
    }
    return t;
}

// 16 bytes a lane from memory into LDS, to 16 lane bytes behind `to`; zeros for what lies behind the buffer's end.  The compiler does not wait for what
// these bring before it reads LDS: wait_loads and meet do.
__device__ __forceinline__ void load_to_lds(Rsrc buffer, uint32_t at, uint32_t to) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(buffer, (__attribute__((address_space(3))) void*)(uintptr_t)to, 16, (int)at, 0, 0, 0);
}
template <int N> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
// The wavefront's accesses to LDS are done, and so are everyone's.
__device__ __forceinline__ void meet() {
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}
__device__ __forceinline__ Rsrc buffer_of(const char* p, uint32_t bytes) {
    const uint64_t at = (uint64_t)p;
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)at), hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(at >> 32));
    return __builtin_amdgcn_make_buffer_rsrc((void*)((uint64_t)hi << 32 | lo), 0, __builtin_amdgcn_readfirstlane((int)bytes), 0x00027000);
}
constexpr uint32_t kNowhere = 0x80000000u;  // behind the end of any buffer here

constexpr int kXcds = 8, kStrip = 4;  // tiles of rows that are walked together

// DIRECT: the tiles go from memory into LDS without passing through registers, which needs whole vectors of sixteen bytes: aligned rows, and widths of a multiple
// of eight.  The other form takes any.
template <class T, bool TRANSPOSED, bool DIRECT>
__global__ __launch_bounds__(T::kThreads) void apm_product_kernel(ProductArgs a) {
    constexpr int FM = T::FM, FN = T::FN, S = T::kStages, kSteps = T::K / kStep;
    static_assert(kSteps % 2 == 0, "two sets of fragments");
    __shared__ __attribute__((aligned(1024))) char lds_all[S * T::kStage];
    lds_char* const lds = (lds_char*)lds_all;
    const int tid = (int)threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);

    // Which tile.  Workgroups go to the XCDs in turn; each XCD takes a stretch of the order, in which tiles come strip by strip.
    int64_t begin = 0, end = a.tokens;
    int group = 0;
    uint32_t row_tile, n_tile;
    {
        uint32_t rows = 0;
        if (a.offsets) {
            for (int g = 0; g < a.groups; g += kWave) rows += (uint32_t)__builtin_amdgcn_readlane((int)tiles_up_to<T::kM>(a, g, lane), kWave - 1);
        } else {
            rows = (uint32_t)((a.tokens + T::kM - 1) / T::kM);
        }
        const uint32_t tiles = rows * (uint32_t)a.tiles_n, nth = blockIdx.x;
        if (nth >= tiles) return;
        const uint32_t xcd = nth % kXcds, id = xcd * (tiles / kXcds) + min(xcd, tiles % kXcds) + nth / kXcds;
        const uint32_t strip = id / (uint32_t)(kStrip * a.tiles_n), in_strip = id - strip * (uint32_t)(kStrip * a.tiles_n), high = min((uint32_t)kStrip, rows - strip * kStrip);
        row_tile = strip * kStrip + in_strip % high, n_tile = in_strip / high;
        if (a.offsets) {
            uint32_t before = 0;
            for (int g = 0; g < a.groups; g += kWave) {
                const uint32_t up = before + tiles_up_to<T::kM>(a, g, lane);
                const uint64_t further = __ballot(up > row_tile);
                if (further) {
                    const int l = __builtin_ctzll(further);
                    group = g + l;
                    row_tile -= l > 0 ? (uint32_t)__builtin_amdgcn_readlane((int)up, l - 1) : before;
                    break;
                }
                before = (uint32_t)__builtin_amdgcn_readlane((int)up, kWave - 1);
            }
            group = __builtin_amdgcn_readfirstlane(group);
            row_tile = (uint32_t)__builtin_amdgcn_readfirstlane((int)row_tile);
            group_of(a, group, &begin, &end);
        }
    }
    const int64_t m0 = begin + (int64_t)row_tile * T::kM;
    const int n0 = (int)n_tile * T::kN;
    const char* const w = a.w + (int64_t)group * a.w_group_stride * 2;
    const int stages = (a.in + T::K - 1) / T::K;

    // What a lane brings of a stage, vector by vector.
    constexpr int kVecsK = T::K / kVec, kVecsN = T::kN / kVec;
    uint32_t at_a[T::kA], at_b[T::kB];    // DIRECT: bytes from the tile's corner
    int vec_a[T::kA], vec_b[T::kB];       // the vector's place in k
    Rsrc buf_a, buf_b;
    u32x4 ra[T::kA], rb[T::kB];           // otherwise: a stage on its way
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
    auto bring = [&](int j) {  // stage j, DIRECT
        const uint32_t to = lds_base + (uint32_t)(j % S) * T::kStage;
        const int k0 = j * T::K;
        const bool whole = k0 + T::K <= a.in;
#pragma unroll
        for (int i = 0; i < T::kA; ++i) {
            uint32_t at = at_a[i] + (uint32_t)k0 * 2u;
            if (at_a[i] == kNowhere || (!whole && k0 + vec_a[i] * kVec >= a.in)) at = kNowhere;
            load_to_lds(buf_a, at, to + (uint32_t)(wave * T::kA + i) * 1024u);
        }
#pragma unroll
        for (int i = 0; i < T::kB; ++i) {
            uint32_t at;
            if constexpr (TRANSPOSED) {
                at = at_b[i] + (uint32_t)k0 * (uint32_t)a.w_stride * 2u;
                if (!whole && k0 + vec_b[i] >= a.in) at = kNowhere;
            } else {
                at = at_b[i] + (uint32_t)k0 * 2u;
                if (at_b[i] == kNowhere || (!whole && k0 + vec_b[i] * kVec >= a.in)) at = kNowhere;
            }
            load_to_lds(buf_b, at, to + T::kBytesA + (uint32_t)(wave * T::kB + i) * 1024u);
        }
    };
    // Rows behind the group's last and columns behind the matrix's are some other ones: what comes of them is not stored.  Behind the end of k
    // there are zeros, in both operands.
    auto fetch = [&](int j) {
        const int k0 = j * T::K;
        const bool whole = k0 + T::K <= a.in;
#pragma unroll
        for (int i = 0; i < T::kA; ++i) {
            const int place = i * T::kThreads + tid, row = place / kVecsK, k = k0 + place % kVecsK * kVec;
            Raw<bf16> r;
            r.load(a.x + min(m0 + row, end - 1) * a.x_stride * 2, k, whole ? kVec : a.in - k);
            ra[i] = r.a;
        }
#pragma unroll
        for (int i = 0; i < T::kB; ++i) {
            const int place = i * T::kThreads + tid;
            Raw<bf16> r;
            if constexpr (TRANSPOSED) {
                const int k = k0 + place / kVecsN, n = n0 + place % kVecsN * kVec;
                r.load(w + (int64_t)k * a.w_stride * 2, n, k < a.in ? min(kVec, a.out - n) : 0);
            } else {
                const int row = place / kVecsK, k = k0 + place % kVecsK * kVec;
                r.load(w + (int64_t)min(n0 + row, a.out - 1) * a.w_stride * 2, k, whole ? kVec : a.in - k);
            }
            rb[i] = r.a;
        }
    };
    typedef __attribute__((address_space(3))) u32x4* lds_vec;
    auto put = [&](int j) {
        lds_char* const to = lds + j % S * T::kStage;
#pragma unroll
        for (int i = 0; i < T::kA; ++i) {
            const int place = i * T::kThreads + tid;
            *(lds_vec)(to + lds_at<T::K>(place / kVecsK, place % kVecsK)) = ra[i];
        }
#pragma unroll
        for (int i = 0; i < T::kB; ++i) {
            const int place = i * T::kThreads + tid;
            if constexpr (TRANSPOSED) *(lds_vec)(to + T::kBytesA + lds_at_t<T::kN>(place / kVecsN, place % kVecsN)) = rb[i];
            else *(lds_vec)(to + T::kBytesA + lds_at<T::K>(place / kVecsK, place % kVecsK)) = rb[i];
        }
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
        const lds_char* const from = lds + j % S * T::kStage;
#pragma unroll
        for (int m = 0; m < FM; ++m) fa[step % 2][m] = read_fragment<T::K>(from, wm + m, step, lane);
#pragma unroll
        for (int n = 0; n < FN; ++n) {
            if constexpr (TRANSPOSED) fb[step % 2][n] = read_fragment_t<T::kN>(from + T::kBytesA, wn + n, step, lane);
            else fb[step % 2][n] = read_fragment<T::K>(from + T::kBytesA, wn + n, step, lane);
        }
    };
    constexpr int kLoads = T::kA + T::kB;
    if constexpr (DIRECT) {
#pragma unroll
        for (int j = 0; j < S; ++j)
            if (j < stages) bring(j);
        if (S <= stages) wait_loads<(S - 1) * kLoads>();
        else wait_loads<0>();
    } else {
#pragma unroll
        for (int j = 0; j < S; ++j)
            if (j < stages) fetch(j), put(j);
        if (S < stages) fetch(S);
    }
    meet();
    read(0, 0);
    // A stage, in steps.  Fragments are read a step ahead; before the last step everybody has read this stage, whose place is filled anew, and the
    // next stage is there.
    for (int j = 0; j < stages; ++j) {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const bool last = s == kSteps - 1;
            if (last) {
                if constexpr (DIRECT) {
                    if (j + S <= stages) wait_loads<(S - 2) * kLoads>();
                    else wait_loads<0>();
                }
                meet();
                if (j + S < stages) {
                    if constexpr (DIRECT) {
                        bring(j + S);
                    } else {
                        put(j + S);
                        if (j + S + 1 < stages) fetch(j + S + 1);
                    }
                }
            }
            read(last ? j + 1 : j, (s + 1) % kSteps);
#pragma unroll
            for (int m = 0; m < FM; ++m)
#pragma unroll
                for (int n = 0; n < FN; ++n) acc[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[s % 2][m], fb[s % 2][n], acc[m][n], 0, 0, 0);
        }
    }
    meet();

    // Lane l has column l mod 32 of a fragment's tile, rows 8 (r / 4) + 4 (l / 32) + r mod 4 in register r.  Rows are stored in whole vectors: half a fragment's
    // rows at a time go through LDS, each wavefront for itself.
    constexpr int kRow = FN * kFrag + 4, kPer = FN * kFrag / kVec, kRowsAtOnce = kWave / kPer;
    static_assert(T::kWaves * 16 * kRow * 4 <= S * T::kStage, "the wavefronts' rows fit");
    typedef __attribute__((address_space(3))) float lds_float;
    lds_float* const mine = (lds_float*)lds + wave * 16 * kRow;
    const int c = lane % kPer * kVec, col = n0 + wn * kFrag + c, there = max(0, min(kVec, a.out - col));
    const int size = a.y_type == APM_F32 ? 4 : 2;
    float bias[kVec] = {};
    if (a.bias.data) {
        RawAny raw;
        const int64_t first = (int64_t)group * a.out + (there > 0 ? col : 0);
        raw.load((const char*)a.bias.data + first * (a.bias.dtype == APM_F32 ? 4 : 2), a.bias.dtype, 0, there);
        raw.get(a.bias.dtype, bias);
    }
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
                const int n = t < end ? there : 0;
                char* to = a.y + t * a.y_stride * size;
                float v[kVec];
#pragma unroll
                for (int e = 0; e < kVec; ++e) v[e] = mine[row * kRow + c + e] + bias[e];
                if (a.accumulate) {
                    RawAny old;
                    old.load(to, a.y_type, n > 0 ? col : 0, n);
                    float f[kVec];
                    old.get(a.y_type, f);
#pragma unroll
                    for (int e = 0; e < kVec; ++e) v[e] += f[e];
                }
                if (a.y_type == APM_F32) store8<float>(to, col, n, v);
                else store8<bf16>(to, col, n, v);
            }
        }
}

int check_product(const apm_grouped_product_desc& p) {
    if (p.tokens < 0 || p.tokens > ((int64_t)1 << 40) || p.out < 1 || p.in < 1 || p.out > kMostCols || p.in > kMostCols || p.n_groups < 0 || p.n_groups > APM_MAX_POSITIONS)
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

enum { kLarge, kSmall, kTiny, kThin };
struct ProductShape {
    int which;
    bool direct;
    int64_t tiles_m, tiles_n;
};
template <class T> void shape_as(const apm_grouped_product_desc& p, int which, ProductShape* s) {
    s->which = which;
    // tokens fill whole tiles but for the last of each group
    const int64_t groups = std::max<int64_t>(1, p.n_groups);
    s->tiles_m = std::min(p.tokens, p.tokens / T::kM + std::min(groups, p.tokens));
    s->tiles_n = div_up(p.out, T::kN);
}
ProductShape product_shape(const apm_grouped_product_desc& p) {
    ProductShape s{};
    const int64_t groups = std::max<int64_t>(1, p.n_groups), each = p.tokens / groups;
    if (each > 128) shape_as<Large>(p, kLarge, &s);
    else if (each > 64) shape_as<Small>(p, kSmall, &s);
    else if (each > 32) shape_as<Tiny>(p, kTiny, &s);
    else shape_as<Thin>(p, kThin, &s);
    const int64_t reach = (int64_t)1 << 30, w_rows = p.transposed ? p.in + Large::K * Large::kStages : Large::kN;
    s.direct = aligned_to(p.x.data, 16) && aligned_to(p.w.data, 16) && p.x.stride % kVec == 0 && p.w.stride % kVec == 0 && (p.n_groups < 2 || p.w_group_stride % kVec == 0) &&
               p.in % kVec == 0 && (!p.transposed || p.out % kVec == 0) && p.x.stride < reach / Large::kM && p.w.stride < reach / w_rows && p.in < reach / 4 && p.out < reach / 4;
    return s;
}

template <class T> hipError_t launch_product(const ProductArgs& a, bool transposed, bool direct, unsigned workgroups, hipStream_t s) {
    auto start = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(workgroups), dim3(T::kThreads), 0, s, a); };
    if (transposed) direct ? start(apm_product_kernel<T, true, true>) : start(apm_product_kernel<T, true, false>);
    else direct ? start(apm_product_kernel<T, false, true>) : start(apm_product_kernel<T, false, false>);
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
    const ProductShape s = product_shape(p);
    a.tiles_n = (int32_t)s.tiles_n;
    if (s.tiles_m > max_workgroups(Large::kThreads) / s.tiles_n) return fail(APM_EINVAL, "y is too large for one product");
    const unsigned n = (unsigned)(s.tiles_m * s.tiles_n);
    const hipStream_t st = (hipStream_t)stream;
    APM_HIP(s.which == kLarge   ? launch_product<Large>(a, p.transposed, s.direct, n, st)
            : s.which == kSmall ? launch_product<Small>(a, p.transposed, s.direct, n, st)
            : s.which == kTiny  ? launch_product<Tiny>(a, p.transposed, s.direct, n, st)
                                : launch_product<Thin>(a, p.transposed, s.direct, n, st));
    return APM_OK;
}

}  // namespace
}  // namespace apm

extern "C" size_t apm_grouped_product_workspace_bytes(const apm_grouped_product_desc*) { return 0; }

extern "C" int apm_grouped_product(const apm_grouped_product_desc* p, void* workspace, size_t workspace_bytes, void* stream) {
    return apm::guarded([&]() -> int { return apm::grouped_product(p, workspace, workspace_bytes, stream); });
}
