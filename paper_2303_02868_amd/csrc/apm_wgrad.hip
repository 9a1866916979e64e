// Weight gradients of linear layers whose input was kept in 8 bits: dw[o, k] = sum over tokens of dy[t, o] z[t, k], one product or one
// for each group of tokens.  On the matrix cores: the kept bytes become bf16 on their way into LDS, which is exact (a whole number of
// seven bits, or a float of four, times a power of two; below 2^-126 it may become zero), so products are exact and sums are fp32.  What the norm in front of the
// layer multiplies and adds per column enters after the sum: z = hat w + b gives (dy^T hat) w + (sum of dy) b.
//
// Both operands lie in memory with the tokens, over which is summed, as rows, so neither has the order that the matrix
// instructions take: tiles go into LDS as they lie and are read with the transposing loads, four tokens of a column at a time.
#include <algorithm>

#include "apm_act.h"

namespace apm {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kWave = 64;
constexpr int kFrag = 32, kStep = 16;  // a matrix instruction's tile, and the tokens that it takes

// A workgroup's tile of dw: WO x WK wavefronts of FO x FK fragments, 64 tokens at a time.  What comes from memory for a later tile of
// tokens waits in DEPTH sets of registers.
template <int WO_, int WK_, int FO_, int FK_, int DEPTH_>
struct Tile {
    static constexpr int WO = WO_, WK = WK_, FO = FO_, FK = FK_, kDepth = DEPTH_, kTokens = 64;
    static constexpr int kOut = WO * FO * kFrag, kIn = WK * FK * kFrag, kThreads = WO * WK * kWave;
    static constexpr int kA = kTokens * kOut / kVec / kThreads;       // vectors of dy that a thread brings
    static constexpr int kB = kTokens * kIn / (2 * kVec) / kThreads;  // 16 kept bytes each
};
// 256 x 256: a byte that comes in is used most often, and one workgroup fills a CU's registers.  128 x 128: four times as many tiles, for small
// dw; one set of registers more hides what the shorter work on a tile does not (256 x 256 over 16384 tokens by one workgroup each, us: 206
// with one set, 184 with two).
typedef Tile<4, 2, 2, 4, 1> Large;
typedef Tile<4, 2, 1, 2, 2> Small;
// 64 x 64, of which four share a CU: the shortest way from the first load to the last store (1000 tokens x 768 x 768 to fp32, without sums 11.3 us, by
// 128 x 128 in two parts 16.5).
// With one set of registers for later tiles 11.6 us there, and 2048 x 768 x 2304 (F8) 21.2 instead of 19.5; 64 tokens take 0.3 us more with two.
typedef Tile<2, 2, 1, 1, 2> Tiny;

struct WgradArgs {
    const char* dy;
    const char* q;
    const uint8_t* scale;
    const int64_t* offsets;
    apm_vector weight, bias, db;
    char* dw;
    float* part;   // [splits][groups][out][in], and sums of dy [splits][groups][out] behind, if splits > 1
    float* sums;
    int64_t dy_stride, q_stride, scale_stride, dw_stride, group_stride;
    int64_t tokens, out, in;
    int32_t groups, splits, tiles_in, tiles;
    int32_t first_group;
    int32_t near_rows;  // rows lie so near to each other that a tile's addresses are 32-bit offsets
    int32_t dw_type, accumulate;
};

// LDS: the 64-byte chunks of a tile's row t are exchanged by t mod 4 (or, where a row is two of them and two rows fill the banks, by half of that), so that
// the four rows that a transposing load takes a chunk of lie in different banks.
template <int ROW> __device__ __forceinline__ int exchange(int t) { return ROW >= 256 ? t & 3 : (t >> 1) & 1; }
template <int ROW> __device__ __forceinline__ int lds_at(int t, int byte) { return t * ROW + ((((byte >> 6) ^ exchange<ROW>(t)) << 6) | (byte & 63)); }

// A fragment of one operand: lane l gets column l mod 32, eight tokens from 8 (l / 32) on.  A transposing load gives each of 16 lanes a column of
// four rows that they bring together, eight bytes each.
template <int ROW> __device__ __forceinline__ bf16x8 read_fragment(const char* tile, int frag, int t0, int lane) {
    typedef __attribute__((address_space(3))) s16x4* lds_ptr;
    const int row = t0 + 8 * (lane / 32) + (lane % 16) / 4;
    const char* p = tile + row * ROW + ((frag ^ exchange<ROW>(row)) << 6) + ((lane / 16) & 1) * 32 + (lane & 3) * 8;
    union {
        s16x4 h[2];
        bf16x8 v;
    } u;
    u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)p);
    u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p + 4 * ROW));
    return u.v;
}

// Eight kept bytes as bf16.
__device__ __forceinline__ u32x4 to_bf16x8(u32x2 q, uint32_t s, int32_t format) {
    u32x4 w;
    if (format == APM_CKPT_I8) {
        float v[kVec];
        decode8(q, scale_of(s, APM_CKPT_I8), APM_CKPT_I8, v);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = to_bf16x2(v[2 * i], v[2 * i + 1]);
    } else {
        const float m = __builtin_bit_cast(float, s << 23);  // the instruction takes the exponent's byte alone, 255 for NaN
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            w[2 * h] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q[h], m, false));
            w[2 * h + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q[h], m, true));
        }
    }
    return w;
}

__device__ __forceinline__ void tokens_of(const WgradArgs& a, int64_t group, int64_t* begin, int64_t* end) {
    *begin = 0, *end = a.tokens;
    if (!a.offsets) return;
    *begin = min(max(a.offsets[group], (int64_t)0), a.tokens);
    *end = min(max(a.offsets[group + 1], *begin), a.tokens);
}

__device__ __forceinline__ void finish_sum(const WgradArgs& a, int64_t group, int64_t o, float sum) {
    const int64_t at = group * a.out + o;
    if (a.accumulate) sum += load1(a.db.data, a.db.dtype, at);
    store1(a.db.data, a.db.dtype, at, sum);
}
// Eight sums of row o from column k on, n of them there, become dw: v weight + bias (sum of dy), added to what is there if asked for. Where the bias is
// zero, as it is where there is none, no sum of dy is added: it may be an infinity where dw is a number.
struct Columns {
    float w[kVec], b[kVec];
    __device__ __forceinline__ void load(const WgradArgs& a, int64_t k, int n, bool with_bias) {
        const int64_t at = n > 0 ? k : 0;
        RawAny raw;
#pragma unroll
        for (int e = 0; e < kVec; ++e) w[e] = 1.0f, b[e] = 0.0f;
        if (a.weight.data) {
            raw.load(a.weight.data, a.weight.dtype, (int)at, n);
            raw.get(a.weight.dtype, w);
        }
        if (with_bias && a.bias.data) {
            raw.load(a.bias.data, a.bias.dtype, (int)at, n);
            raw.get(a.bias.dtype, b);
        }
    }
};
// HOP > 0: the lanes' upper half has the rows HOP below those of the lower half, and if `whole` all 64 have eight columns of a row.
template <int HOP>
__device__ __forceinline__ void finish(const WgradArgs& a, const Columns& c, int64_t group, int64_t o, int64_t k, int n, bool whole, float (&v)[kVec], float sum) {
    char* row = a.dw + (group * a.group_stride + o * a.dw_stride) * (a.dw_type == APM_F32 ? 4 : 2);
#pragma unroll
    for (int e = 0; e < kVec; ++e) v[e] = fmaf(v[e], c.w[e], c.b[e] == 0.0f ? 0.0f : c.b[e] * sum);
    if (a.accumulate) {
        RawAny old;
        old.load(row, a.dw_type, (int)k, n);
        float f[kVec];
        old.get(a.dw_type, f);
#pragma unroll
        for (int e = 0; e < kVec; ++e) v[e] += f[e];
    }
    // fp32 in whole cache lines at a time, the lower half of the lanes' rows, then the upper half's (64 groups of 704 x 2560, a token each: 152 us with a
    // lane's own 32 bytes, so 107).
    if (HOP > 0 && whole && a.dw_type == APM_F32) {
        u32x4 w[2];
#pragma unroll
        for (int e = 0; e < kVec; ++e) w[e / 4][e % 4] = __builtin_bit_cast(uint32_t, v[e]);
        swap_halves(w[0], w[1]);
        const int64_t hop = HOP * a.dw_stride * 4;
        const bool upper = threadIdx.x % kWave >= kWave / 2;
        char* at = row + k * 4 + (upper ? 16 : 0);
        store_at<true>(w[0], (u32x4_any*)(at - (upper ? hop : 0)));
        store_at<true>(w[1], (u32x4_any*)(at + (upper ? 0 : hop)));
        return;
    }
    if (a.dw_type == APM_F32) store8<float, true>(row, (int)k, n, v);
    else store8<bf16, true>(row, (int)k, n, v);
}

// What lanes of a wavefront hand each other through LDS: its accesses are carried out in order, so it is the compiler's order that counts.
__device__ __forceinline__ void among_lanes() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

constexpr int kXcds = 8;
constexpr int kStrip = 4;  // rows of tiles that are walked together

// 16384 tokens x 8192 x 2048: 495 us = 1110 TFLOP/s (I8), 483 (F8), with sums 536 and 533; a library product of bf16 matrices in this order 480, in the
// order that suits it 369 (on another card 475, 507 with sums, and 462).  No unit alone bounds it: of a CU's cycles the matrix cores are busy for 54 %, other
// vector instructions issue for 35 %, LDS works for 41 % (with transposing loads, which give about 120 bytes a clock, and a sixth of it conflicts), and
// two wavefronts a SIMD overlap them in part.
template <class T, int FORMAT, bool SUMS>
__global__ __launch_bounds__(T::kThreads) void apm_wgrad_kernel(WgradArgs a) {
    constexpr int kRowA = T::kOut * 2, kRowB = T::kIn * 2, kTokens = T::kTokens, FO = T::FO, FK = T::FK, D = T::kDepth, kSteps = kTokens / kStep;
    constexpr int kTileA = kTokens * kRowA, kTileB = kTokens * kRowB;
    __shared__ __attribute__((aligned(16))) char lds[2 * (kTileA + kTileB)];
    __shared__ float row_sum[SUMS ? T::kOut : 1];
    auto tile_a = [&](int buf) -> char* { return lds + buf * kTileA; };
    auto tile_b = [&](int buf) -> char* { return lds + 2 * kTileA + buf * kTileB; };
    const int tid = (int)threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    // Workgroups go to the XCDs in turn.  Each XCD takes a stretch of the order, in which tiles come strip by strip, so that its L2 meets few
    // rows and columns (16384 x 8192 x 2048, TFLOP/s when this was chosen: 930 in launch order, 970 with strips of 4 rows, 920 of 16).
    // Groups one after the other on all XCDs: they have different numbers of tokens.
    const uint32_t in_group = (uint32_t)(a.tiles * a.splits), nth = blockIdx.x % in_group, x = nth % kXcds;
    const uint32_t id = x * (in_group / kXcds) + min(x, in_group % kXcds) + nth / kXcds;
    const int group = a.first_group + (int)(blockIdx.x / in_group), split = (int)(id / (uint32_t)a.tiles), tile = (int)(id % (uint32_t)a.tiles);
    const int strip = tile / (kStrip * a.tiles_in), in_strip = tile - strip * kStrip * a.tiles_in, high = min(kStrip, a.tiles / a.tiles_in - strip * kStrip);
    const int64_t o0 = (int64_t)(strip * kStrip + in_strip % high) * T::kOut, k0 = (int64_t)(in_strip / high) * T::kIn;
    int64_t begin, end;
    tokens_of(a, group, &begin, &end);
    // No sum at all: not even weight times it.  Stored non-temporally, as the results are: rows of other groups stay in L2 (64 groups of 4096 x 1024, an
    // eighth of them with tokens: 181 us, with non-temporal stores 131; zeros alone 97).  In fp32 with eight elements a lane, which halves of lines take,
    // 64 empty groups of 704 x 2560 took 194 us, so 91.
    if (begin == end && a.splits == 1) {
        if (a.accumulate) return;
        const bool wide = a.dw_type == APM_F32;
        const int size = wide ? 4 : 2, per = 16 / size, in_row = T::kIn / per;  // 16 bytes a lane, next to its neighbours' in both types
#pragma unroll 4
        for (int i = tid; i < T::kOut * in_row; i += T::kThreads) {
            const int64_t o = o0 + i / in_row, k = k0 + i % in_row * per;
            char* to = a.dw + (group * a.group_stride + o * a.dw_stride + k) * size;
            if (o >= a.out) continue;
            if (k + per <= a.in) {
                store_at<true>(u32x4{0u, 0u, 0u, 0u}, (u32x4_any*)to);
            } else {
                for (int64_t e = k; e < a.in; ++e, to += size) {
                    if (wide) *(uint32_t*)to = 0u;
                    else *(uint16_t*)to = 0;
                }
            }
        }
        if (SUMS && a.db.data && k0 == 0 && tid < T::kOut && o0 + tid < a.out) finish_sum(a, group, o0 + tid, 0.0f);
        return;
    }
    if (a.splits > 1) {
        const int64_t each = (end - begin + (int64_t)a.splits * kTokens - 1) / ((int64_t)a.splits * kTokens) * kTokens;
        begin = min(begin + split * each, end);
        end = min(begin + each, end);
    }

    u32x4 sa[D][T::kA] = {}, sb[D][T::kB] = {};
    uint32_t ss[D][T::kB] = {};
    constexpr int kPerRowA = T::kOut / kVec, kRowsA = T::kThreads / kPerRowA, kPerRowB = T::kIn / (2 * kVec), kRowsB = T::kThreads / kPerRowB;
    const int row_a = tid / kPerRowA, col_a = tid % kPerRowA * kVec, row_b = tid / kPerRowB, col_b = tid % kPerRowB * 2 * kVec;
    // Whole tiles of tokens whose loads end inside the matrices; columns beyond a tile's edge then are the next row's, and land in what is not stored.
    auto load = [&](int set, int64_t t0) {
        const char* pa = a.dy + (t0 * a.dy_stride + o0) * 2;
        const char* pq = a.q + t0 * a.q_stride + k0;
        const uint8_t* ps = a.scale + t0 * a.scale_stride + k0 / APM_CKPT_BLOCK;
        const uint32_t da = ((uint32_t)row_a * (uint32_t)a.dy_stride + (uint32_t)col_a) * 2u, dq = (uint32_t)row_b * (uint32_t)a.q_stride + (uint32_t)col_b,
                       ds = (uint32_t)row_b * (uint32_t)a.scale_stride + (uint32_t)col_b / APM_CKPT_BLOCK;
#pragma unroll
        for (int i = 0; i < T::kA; ++i) sa[set][i] = *(const u32x4_any*)(pa + i * kRowsA * a.dy_stride * 2 + da);
#pragma unroll
        for (int i = 0; i < T::kB; ++i) {
            sb[set][i] = *(const u32x4_any*)(pq + i * kRowsB * a.q_stride + dq);
            ss[set][i] = ps[i * kRowsB * a.scale_stride + ds];
        }
    };
    auto load_guarded = [&](int set, int64_t t0) {
#pragma unroll
        for (int i = 0; i < T::kA; ++i) {
            const int64_t t = t0 + row_a + i * kRowsA, o = o0 + col_a;
            Raw<bf16> r;
            r.load(a.dy + t * a.dy_stride * 2, (int)o, t < end ? (int)min((int64_t)kVec, a.out - o) : 0);
            sa[set][i] = r.a;
        }
#pragma unroll
        for (int i = 0; i < T::kB; ++i) {
            const int64_t t = t0 + row_b + i * kRowsB, k = k0 + col_b;
            const int n = t < end ? (int)min((int64_t)(2 * kVec), a.in - k) : 0;
            const u32x2 lo = load_q(a.q + t * a.q_stride, (int)k, n), hi = load_q(a.q + t * a.q_stride, (int)k + kVec, n - kVec);
            sb[set][i] = u32x4{lo[0], lo[1], hi[0], hi[1]};
            ss[set][i] = n > 0 ? a.scale[t * a.scale_stride + k / APM_CKPT_BLOCK] : 0u;
        }
    };
    auto put_a = [&](int buf, int set, int i) { *(u32x4*)(tile_a(buf) + lds_at<kRowA>(row_a + i * kRowsA, col_a * 2)) = sa[set][i]; };
    auto put_b = [&](int buf, int set, int i) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
            *(u32x4*)(tile_b(buf) + lds_at<kRowB>(row_b + i * kRowsB, (col_b + h * kVec) * 2)) =
                to_bf16x8(u32x2{sb[set][i][2 * h], sb[set][i][2 * h + 1]}, ss[set][i], FORMAT);
    };

    f32x16 acc[FO][FK];
    float sum[FO];
#pragma unroll
    for (int m = 0; m < FO; ++m) {
        sum[m] = 0.0f;
#pragma unroll
        for (int n = 0; n < FK; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[m][n][r] = 0.0f;
    }
    const int wm = wave / T::WK * FO, wn = wave % T::WK * FK;  // the wavefront's first fragments
    // Fragments of dy for two steps; of what was kept for two where registers are left; of both for all steps where a wavefront has one of each, which
    // then waits for LDS once a tile and not at each step (2048 tokens x 1024 x 1024 in F8: 16.6 us, so 16.0; without sums 13.7 and 13.2).
    constexpr bool kWhole = FO * FK == 1;
    constexpr int kSetsA = kWhole ? kSteps : 2, kSetsB = kWhole ? kSteps : FO * FK == 8 ? 1 : 2;
    bf16x8 fa[kSetsA][FO], fb[kSetsB][FK];
    auto read_a = [&](int buf, int step) {
#pragma unroll
        for (int m = 0; m < FO; ++m) fa[step % kSetsA][m] = read_fragment<kRowA>(tile_a(buf), wm + m, step * kStep, lane);
    };
    auto read_b = [&](int buf, int step) {
#pragma unroll
        for (int n = 0; n < FK; ++n) fb[step % kSetsB][n] = read_fragment<kRowB>(tile_b(buf), wn + n, step * kStep, lane);
    };
    auto multiply = [&](int step) {
#pragma unroll
        for (int m = 0; m < FO; ++m) {
#pragma unroll
            for (int n = 0; n < FK; ++n) acc[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[step % kSetsA][m], fb[step % kSetsB][n], acc[m][n], 0, 0, 0);
            if constexpr (SUMS) {
                const bf16x2 one = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
                for (int i = 0; i < kVec; i += 2) sum[m] = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{fa[step % kSetsA][m][i], fa[step % kSetsA][m][i + 1]}, one, sum[m], false);
            }
        }
    };
    // A tile of tokens, in steps.  Fragments are read a step ahead.  In the middle steps what a set of registers holds of the next tile goes into the
    // other buffer; before the last one everybody has read this buffer, so that the set is filled anew and the next tile's first fragments are read.
    auto turn = [&](int buf, int set, auto&& fetch) {
        if constexpr (kWhole) {  // the next tile is put down while this one's fragments are on their way
#pragma unroll
            for (int i = 0; i < T::kA; ++i) put_a(buf ^ 1, set, i);
#pragma unroll
            for (int i = 0; i < T::kB; ++i) put_b(buf ^ 1, set, i);
#pragma unroll
            for (int s = 0; s < kSteps; ++s) multiply(s);
            __syncthreads();
            fetch();
#pragma unroll
            for (int s = 0; s < kSteps; ++s) read_a(buf ^ 1, s), read_b(buf ^ 1, s);
            return;
        }
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            if (s == kSteps - 1) {
                __syncthreads();
                fetch();
            }
            const int from = s == kSteps - 1 ? buf ^ 1 : buf, ahead = (s + 1) % kSteps;
            read_a(from, ahead);
            if constexpr (kSetsB == 2) read_b(from, ahead);
            multiply(s);
            if constexpr (kSetsB == 1) read_b(from, ahead);
            if (s > 0 && s < kSteps - 1) {
#pragma unroll
                for (int i = s - 1; i < T::kA; i += kSteps - 2) put_a(buf ^ 1, set, i);
#pragma unroll
                for (int i = s - 1; i < T::kB; i += kSteps - 2) put_b(buf ^ 1, set, i);
            }
            if constexpr (FO * FK == 8) {  // the order that the scheduler is to keep: between two products a part of everything else
#pragma unroll
                for (int i = 0; i < FO * FK; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // matrix
                    __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);  // LDS reads
                    __builtin_amdgcn_sched_group_barrier(0x002, 6, 0);  // vector arithmetic
                    __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);  // LDS writes
                    __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);  // memory reads
                }
            }
        }
    };
    const int64_t n_tiles = (end - begin + kTokens - 1) / kTokens;
    int64_t whole = 0;  // tiles that `load` may take
    if (a.near_rows) {
        auto reach = [&](int64_t stride, int64_t width, int64_t first, int64_t take) {  // tokens of whose rows `take` columns from `first` on may be read
            const int64_t over = first + take - width;
            return over <= 0 ? a.tokens : stride > 0 ? a.tokens - (over + stride - 1) / stride : (int64_t)0;
        };
        const int64_t last = min(end, min(min(reach(a.dy_stride, a.out, o0, T::kOut), reach(a.q_stride, a.in, k0, T::kIn)),
                                          reach(a.scale_stride, (a.in + APM_CKPT_BLOCK - 1) / APM_CKPT_BLOCK, k0 / APM_CKPT_BLOCK, T::kIn / APM_CKPT_BLOCK)));
        whole = max((last - begin) / kTokens, (int64_t)0);
    }
    auto fetch = [&](int set, int64_t i) {
        if (i < whole) load(set, begin + i * kTokens);
        else if (i < n_tiles) load_guarded(set, begin + i * kTokens);
    };
    if (n_tiles > 0) {  // the last turns put and read what is not used
        fetch(0, 0);
#pragma unroll
        for (int i = 0; i < T::kA; ++i) put_a(0, 0, i);
#pragma unroll
        for (int i = 0; i < T::kB; ++i) put_b(0, 0, i);
#pragma unroll
        for (int i = 1; i <= D; ++i) fetch(i % D, i);
        __syncthreads();
        read_a(0, 0);
        read_b(0, 0);
        if constexpr (kWhole) {
#pragma unroll
            for (int s = 1; s < kSteps; ++s) read_a(0, s), read_b(0, s);
        }
        int64_t i = 0;
        if constexpr (D == 1) {
            int buf = 0;
            for (; i + 2 < whole; ++i, buf ^= 1) turn(buf, 0, [&] { load(0, begin + (i + 2) * kTokens); });
            for (; i < n_tiles; ++i, buf ^= 1) turn(buf, 0, [&] { fetch(0, i + 2); });
        } else {
            for (; i + 4 < whole; i += 2) {
                turn(0, 1, [&] { load(1, begin + (i + 3) * kTokens); });
                turn(1, 0, [&] { load(0, begin + (i + 4) * kTokens); });
            }
            for (; i < n_tiles; i += 2) {
                turn(0, 1, [&] { fetch(1, i + 3); });
                if (i + 1 < n_tiles) turn(1, 0, [&] { fetch(0, i + 4); });
            }
        }
        __syncthreads();
    }

    // Lane l has column l mod 32 of a fragment's tile, rows 8 (r / 4) + 4 (l / 32) + r mod 4 in register r; a row's sum over the tokens of
    // one half of the lanes each.
    const int64_t gs = (int64_t)split * a.groups + group;
    if constexpr (SUMS) {
#pragma unroll
        for (int m = 0; m < FO; ++m) {
            sum[m] += __shfl_xor(sum[m], 32);
            if (wn == 0 && lane < kFrag) {
                row_sum[(wm + m) * kFrag + lane] = sum[m];
                const int64_t o = o0 + (wm + m) * kFrag + lane;
                if (k0 == 0 && o < a.out) {
                    if (a.splits > 1) a.sums[gs * a.out + o] = sum[m];
                    else if (a.db.data) finish_sum(a, group, o, sum[m]);
                }
            }
        }
        __syncthreads();
    }
    if (a.splits > 1) {
#pragma unroll
        for (int m = 0; m < FO; ++m)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int64_t o = o0 + (wm + m) * kFrag + 8 * (r / 4) + 4 * (lane / 32) + r % 4;
                float* row = a.part + (gs * a.out + o) * a.in;
#pragma unroll
                for (int n = 0; n < FK; ++n) {
                    const int64_t k = k0 + (wn + n) * kFrag + lane % 32;
                    if (o < a.out && k < a.in) row[k] = acc[m][n][r];
                }
            }
        return;
    }
    // Rows are stored in whole vectors: half a fragment's rows at a time go through LDS, each wavefront for itself.
    constexpr int kRow = FK * kFrag + 4, kPer = FK * kFrag / kVec, kRowsAtOnce = kWave / kPer;
    static_assert(T::WO * T::WK * 16 * kRow * 4 <= (int)sizeof lds, "the wavefronts' rows fit");
    float* mine = (float*)lds + wave * 16 * kRow;
    const int c = lane % kPer * kVec;
    const int64_t k = k0 + wn * kFrag + c;
    const int there = (int)max((int64_t)0, min((int64_t)kVec, a.in - k));
    const bool whole_tile = o0 + T::kOut <= a.out && k0 + T::kIn <= a.in;
    Columns cols;
    cols.load(a, k, there, SUMS);
#pragma unroll
    for (int m = 0; m < FO; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h) {  // registers 8 h .. 8 h + 7: rows 16 h .. 16 h + 15
            among_lanes();
#pragma unroll
            for (int r = 0; r < 8; ++r)
#pragma unroll
                for (int n = 0; n < FK; ++n) mine[(8 * (r / 4) + 4 * (lane / 32) + r % 4) * kRow + n * kFrag + lane % 32] = acc[m][n][8 * h + r];
            among_lanes();
#pragma unroll
            for (int i = 0; i < 16 / kRowsAtOnce; ++i) {
                const int row = i * kRowsAtOnce + lane / kPer, in_tile = (wm + m) * kFrag + 16 * h + row;
                const int64_t o = o0 + in_tile;
                float v[kVec];
#pragma unroll
                for (int e = 0; e < kVec; ++e) v[e] = mine[row * kRow + c + e];
                finish<kRowsAtOnce / 2>(a, cols, group, o, k, o < a.out ? there : 0, whole_tile, v, SUMS ? row_sum[in_tile] : 0.0f);
            }
        }
}

// The splits' parts, added in order: eight columns of a row a thread, four parts under way at a time.
constexpr int kJoinThreads = 256;
template <bool SUMS>
__global__ __launch_bounds__(kJoinThreads) void apm_wgrad_join_kernel(WgradArgs a) {
    const uint32_t per_row = (uint32_t)((a.in + kVec - 1) / kVec), id = blockIdx.x * kJoinThreads + threadIdx.x, row = id / per_row;
    const int64_t rows = (int64_t)a.groups * a.out;
    if (row >= rows) return;
    const int k = (int)(id - row * per_row) * kVec, n = (int)min((int64_t)kVec, a.in - k);
    const int64_t group = row / (uint32_t)a.out, o = row - (uint32_t)group * (uint32_t)a.out;
    int64_t begin, end;
    tokens_of(a, group, &begin, &end);
    Columns cols;
    cols.load(a, k, begin < end ? n : 0, SUMS);
    float v[kVec] = {}, sum = 0.0f;
    for (int s = 0; s < a.splits; s += 4) {
        Raw<float> part[4];
        float of_row[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            part[i].load(a.part + ((s + i) * rows + row) * a.in, k, s + i < a.splits ? n : 0);
            if constexpr (SUMS) of_row[i] = s + i < a.splits ? a.sums[(s + i) * rows + row] : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (SUMS) sum += of_row[i];
#pragma unroll
            for (int e = 0; e < kVec; ++e) v[e] += part[i][e];
        }
    }
    if (SUMS && k == 0 && a.db.data) finish_sum(a, group, o, sum);
    finish<0>(a, cols, group, o, k, n, false, v, sum);
}

// Which tile, and into how many parts the tokens are split, so that few tiles fill the chip.  Estimated in us, from calls that were timed: a round of
// workgroups costs `start`, and `turn` for each 64 tokens, or `busy` times the workgroups that share a CU where that is more (with sums; 256 x 256 alone on a CU:
// 534 us for 256 turns, 140 for 64, 14.4 for one; 128 x 128 alone: 205 for 256, 18.4 for 16; 64 x 64 alone: 105 for 256, 12.7 for 16, four on a CU 44 for 32).
// Parts are written and read at 4 TB/s, by one kernel more.  With one part and with several (tokens x out x in): 8192 x 768 x 768 97 / 28, 16384 x 256 x 256 by
// 64 x 64 105 / 22, by 128 x 128 184 with one; 8192 x 2048 x 2048 by 256 x 256 212 / 91, by 128 x 128 103 / 117.  The constants are from an earlier state of the
// tiles: they take a turn of 64 x 64 for 0.55 us, which is 0.41, and 256 x 256 in four parts for slower than 128 x 128 at the last size, where it is faster.
constexpr int64_t kCus = 256, kMostSplits = 64;
enum { kLarge, kSmall, kTiny };
struct WgradShape {
    int which;
    int64_t tiles_out, tiles_in, groups;
    int32_t splits;
    double cost;
};
template <class T>
void best_split(const apm_weight_grad& w, int which, int64_t per_cu, double start, double turn, double busy, WgradShape* best) {
    WgradShape s{which, div_up(w.out, T::kOut), div_up(w.in, T::kIn), std::max<int64_t>(1, w.n_groups), 1, 0.0};
    const int64_t tiles = s.tiles_out * s.tiles_in * s.groups, each = div_up(w.tokens, s.groups);
    for (int64_t n = 1; n <= kMostSplits && (n == 1 || (tiles * n <= 2 * kCus && n <= div_up(each, 2 * T::kTokens))); ++n) {
        const double rounds = (double)div_up(tiles * n, kCus * per_cu), turns = (double)div_up(div_up(each, n), T::kTokens);
        const double parts = n > 1 ? 4.0 + 8.0 * (double)n * (double)s.groups * (double)w.out * (double)w.in / 4e6 : 0.0;
        s.splits = (int32_t)n;
        s.cost = rounds * start + turns * std::max(rounds * turn, busy * (double)(tiles * n) / (double)kCus) + parts;
        if (best->cost < 0.0 || s.cost < best->cost) *best = s;
    }
}
WgradShape wgrad_shape(const apm_weight_grad& w) {
    WgradShape s{kLarge, 0, 0, 0, 1, -1.0};
    best_split<Large>(w, kLarge, 1, 14.0, 1.95, 0.0, &s);
    best_split<Small>(w, kSmall, 1, 8.0, 0.7, 0.0, &s);
    best_split<Tiny>(w, kTiny, 4, 5.0, 0.55, 0.33, &s);
    return s;
}
size_t workspace_of(const apm_weight_grad& w, const WgradShape& s) {
    return s.splits > 1 ? (size_t)s.splits * s.groups * w.out * (w.in + 1) * sizeof(float) : 0;
}

template <class T>
hipError_t launch_wgrad(const WgradArgs& a, int32_t format, bool sums, unsigned workgroups, hipStream_t s) {
    auto start = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(workgroups), dim3(T::kThreads), 0, s, a); };
    if (format == APM_CKPT_I8) sums ? start(apm_wgrad_kernel<T, APM_CKPT_I8, true>) : start(apm_wgrad_kernel<T, APM_CKPT_I8, false>);
    else sums ? start(apm_wgrad_kernel<T, APM_CKPT_F8, true>) : start(apm_wgrad_kernel<T, APM_CKPT_F8, false>);
    return hipGetLastError();
}

int check_grad(const apm_weight_grad& w) {
    if (w.tokens < 0 || w.out < 1 || w.in < 1 || w.out > INT32_MAX / 2 || w.in > INT32_MAX / 2 || w.n_groups < 0 || w.n_groups > INT32_MAX)
        return fail(APM_EINVAL, "bad size: %lld tokens, %lld x %lld, %lld groups", (long long)w.tokens, (long long)w.out, (long long)w.in, (long long)w.n_groups);
    if ((w.n_groups > 0) != (w.offsets != nullptr)) return fail(APM_EINVAL, "offsets and n_groups contradict each other");
    if ((uintptr_t)w.offsets % 8 != 0) return fail(APM_EINVAL, "offsets are not aligned to their elements");
    int rc = check_matrix("dy", w.dy, w.tokens, w.out, false);
    if (rc == APM_OK && w.tokens > 0 && w.dy.dtype != APM_BF16) rc = fail(APM_EINVAL, "dy must be bf16");
    if (rc == APM_OK) rc = check_ckpt("kept", w.kept, w.tokens, w.in, false);
    if (rc == APM_OK) rc = check_vector("weight", w.weight);
    if (rc == APM_OK) rc = check_vector("bias", w.bias);
    if (rc == APM_OK) rc = check_vector("db", w.db);
    if (rc == APM_OK) rc = check_matrix("dw", w.dw, w.out, w.in, true);
    if (rc == APM_OK && w.n_groups > 1 && w.dw_group_stride > ((int64_t)1 << 56) / w.n_groups) rc = fail(APM_EINVAL, "dw's groups are too far apart");
    if (rc == APM_OK && w.n_groups > 1 && w.dw_group_stride < (w.out - 1) * w.dw.stride + w.in) rc = fail(APM_EINVAL, "dw's groups overlap");
    return rc;
}

int weight_grad(const apm_weight_grad* wp, void* workspace, size_t workspace_bytes, void* stream) {
    if (!wp) return fail(APM_EINVAL, "missing argument");
    const apm_weight_grad& w = *wp;
    int rc = check_grad(w);
    if (rc != APM_OK) return rc;
    const WgradShape s = wgrad_shape(w);
    const size_t need = workspace_of(w, s);
    if (workspace_bytes < need) return fail(APM_ENOMEM, "the workspace is too small");
    if (need > 0 && (!workspace || (uintptr_t)workspace % 16 != 0)) return fail(APM_EINVAL, "the workspace is missing or not aligned to 16 bytes");
    WgradArgs a{};
    a.dy = (const char*)w.dy.data, a.q = (const char*)w.kept.q, a.scale = (const uint8_t*)w.kept.scale, a.offsets = w.offsets;
    a.weight = w.weight, a.bias = w.bias, a.db = w.db, a.dw = (char*)w.dw.data;
    a.part = (float*)workspace, a.sums = a.part + (int64_t)s.splits * s.groups * w.out * w.in;
    a.dy_stride = w.dy.stride, a.q_stride = w.kept.q_stride, a.scale_stride = w.kept.scale_stride;
    a.dw_stride = w.dw.stride, a.group_stride = w.dw_group_stride;
    a.tokens = w.tokens, a.out = w.out, a.in = w.in;
    a.groups = (int32_t)s.groups, a.splits = s.splits, a.tiles_in = (int32_t)s.tiles_in;
    a.near_rows = std::max({w.dy.stride, w.kept.q_stride, w.kept.scale_stride}) < (1 << 24);
    a.dw_type = w.dw.dtype, a.accumulate = w.accumulate;
    const int64_t tiles = s.tiles_out * s.tiles_in, most = max_workgroups(std::max({Large::kThreads, Small::kThreads, Tiny::kThreads}));
    if (tiles > most / s.splits) return fail(APM_EINVAL, "dw is too large for one product");
    a.tiles = (int32_t)tiles;
    const bool sums = w.bias.data || w.db.data;
    const hipStream_t st = (hipStream_t)stream;
    const int64_t groups_per_launch = most / (tiles * s.splits);
    for (int64_t g = 0; g < s.groups; g += groups_per_launch) {
        a.first_group = (int32_t)g;
        const unsigned n = (unsigned)(tiles * s.splits * std::min(groups_per_launch, s.groups - g));
        APM_HIP(s.which == kLarge   ? launch_wgrad<Large>(a, w.kept.format, sums, n, st)
                : s.which == kSmall ? launch_wgrad<Small>(a, w.kept.format, sums, n, st)
                                    : launch_wgrad<Tiny>(a, w.kept.format, sums, n, st));
    }
    if (s.splits > 1) {  // so that there are few tiles: under 2^32 vectors
        const dim3 grid((unsigned)div_up(div_up(w.in, kVec) * s.groups * w.out, kJoinThreads));
        if (sums) hipLaunchKernelGGL(apm_wgrad_join_kernel<true>, grid, dim3(kJoinThreads), 0, st, a);
        else hipLaunchKernelGGL(apm_wgrad_join_kernel<false>, grid, dim3(kJoinThreads), 0, st, a);
        APM_HIP(hipGetLastError());
    }
    return APM_OK;
}

}  // namespace
}  // namespace apm

extern "C" size_t apm_ckpt_weight_grad_workspace_bytes(const apm_weight_grad* w) {
    if (!w || apm::check_grad(*w) != APM_OK) return 0;
    return apm::workspace_of(*w, apm::wgrad_shape(*w));
}

extern "C" int apm_ckpt_weight_grad(const apm_weight_grad* w, void* workspace, size_t workspace_bytes, void* stream) {
    return apm::guarded([&]() -> int { return apm::weight_grad(w, workspace, workspace_bytes, stream); });
}

extern "C" int apm_test_weight_grad_tile(const apm_weight_grad* w) {
    constexpr int kSide[] = {apm::Large::kOut, apm::Small::kOut, apm::Tiny::kOut};
    return !w || apm::check_grad(*w) != APM_OK ? 0 : kSide[apm::wgrad_shape(*w).which];
}
