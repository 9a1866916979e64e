// Weight gradients of linear layers whose input was kept in 8 bits: dw[o, k] = sum over tokens of dy[t, o] z[t, k], one product or one
// for each group of tokens.  On the matrix cores: the kept bytes become bf16 on their way into LDS, which is exact (a whole number of
// seven bits, or a float of four, times a power of two), so products are exact and sums are fp32.  What the norm in front of the
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

constexpr int kThreads = 256, kWave = 64;
constexpr int kTile = 128, kTokens = 32;  // a workgroup's tile of dw, and the tokens that it takes at a time
constexpr int kFrag = 32;                 // a matrix instruction's tile, over 16 tokens
constexpr int kPerWave = kTile / 2 / kFrag;
constexpr int kRowBytes = kTile * 2;

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
    int32_t format, dw_type, accumulate;
};

// LDS: row t of a tile is kRowBytes, its 64-byte chunks exchanged by t mod 4, so that the four rows that a transposing load
// takes a chunk of lie in different banks.
__device__ __forceinline__ int lds_at(int t, int byte) { return t * kRowBytes + ((((byte >> 6) ^ (t & 3)) << 6) | (byte & 63)); }

struct Stage {
    u32x4 a[2];
    u32x2 b[2];
    uint32_t s;
    int b_row;
};

__device__ __forceinline__ bf16x8 read_fragment(const char* tile, int frag, int t0, int lane) {
    typedef __attribute__((address_space(3))) s16x4* lds_ptr;
    const int row = t0 + 8 * (lane / 32) + (lane % 16) / 4;
    const char* p = tile + row * kRowBytes + ((frag ^ (row & 3)) << 6) + ((lane / 16) & 1) * 32 + (lane & 3) * 8;
    union {
        s16x4 h[2];
        bf16x8 v;
    } u;
    u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)p);
    u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p + 4 * kRowBytes));
    return u.v;
}

__device__ __forceinline__ void finish(const WgradArgs& a, int64_t group, int64_t o, int64_t k, float v, float sum) {
    if (a.weight.data) v *= load1(a.weight.data, a.weight.dtype, k);
    if (a.bias.data) v = fmaf(load1(a.bias.data, a.bias.dtype, k), sum, v);
    const int64_t at = group * a.group_stride + o * a.dw_stride + k;
    if (a.accumulate) v += load1(a.dw, a.dw_type, at);
    store1(a.dw, a.dw_type, at, v);
}
__device__ __forceinline__ void finish_sum(const WgradArgs& a, int64_t group, int64_t o, float sum) {
    const int64_t at = group * a.out + o;
    if (a.accumulate) sum += load1(a.db.data, a.db.dtype, at);
    store1(a.db.data, a.db.dtype, at, sum);
}

template <bool SUMS>
__global__ __launch_bounds__(kThreads) void apm_wgrad_kernel(WgradArgs a) {
    __shared__ __attribute__((aligned(16))) char tile_a[2][kTokens * kRowBytes], tile_b[2][kTokens * kRowBytes];
    const int tid = (int)threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int tile = (int)(blockIdx.x % (uint32_t)a.tiles), rest = (int)(blockIdx.x / (uint32_t)a.tiles);
    const int split = rest % a.splits, group = a.first_group + rest / a.splits;
    const int64_t o0 = (int64_t)(tile / a.tiles_in) * kTile, k0 = (int64_t)(tile % a.tiles_in) * kTile;
    int64_t begin = 0, end = a.tokens;
    if (a.offsets) {
        begin = min(max(a.offsets[group], (int64_t)0), a.tokens);
        end = min(max(a.offsets[group + 1], begin), a.tokens);
    }
    if (a.splits > 1) {
        const int64_t each = (end - begin + (int64_t)a.splits * kTokens - 1) / ((int64_t)a.splits * kTokens) * kTokens;
        begin = min(begin + split * each, end);
        end = min(begin + each, end);
    }

    auto load = [&](Stage& s, int64_t t0) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int id = i * kThreads + tid, row = id / (kTile / kVec), c = id % (kTile / kVec) * kVec;
            const int64_t t = t0 + row;
            Raw<bf16> r;
            r.load(a.dy + t * a.dy_stride * 2, (int)(o0 + c), t < end ? (int)min((int64_t)kVec, a.out - (o0 + c)) : 0);
            s.a[i] = r.a;
        }
        const int row = tid / 8, c = tid % 8 * 16;
        const int64_t t = t0 + row;
        const int n = t < end ? (int)min((int64_t)16, a.in - (k0 + c)) : 0;
        s.b[0] = load_q(a.q + t * a.q_stride, (int)(k0 + c), n);
        s.b[1] = load_q(a.q + t * a.q_stride, (int)(k0 + c) + kVec, n - kVec);
        s.s = n > 0 ? a.scale[t * a.scale_stride + (k0 + c) / APM_CKPT_BLOCK] : 0u;
    };
    auto put = [&](const Stage& s, int buf) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int id = i * kThreads + tid, row = id / (kTile / kVec), c = id % (kTile / kVec) * kVec;
            *(u32x4*)(tile_a[buf] + lds_at(row, c * 2)) = s.a[i];
        }
        const int row = tid / 8, c = tid % 8 * 16;
        const float m = scale_of(s.s, a.format);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float v[kVec];
            decode8(s.b[h], m, a.format, v);
            u32x4 w;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = to_bf16x2(v[2 * i], v[2 * i + 1]);
            *(u32x4*)(tile_b[buf] + lds_at(row, (c + h * kVec) * 2)) = w;
        }
    };

    f32x16 acc[kPerWave][kPerWave];
    float sum[kPerWave];
#pragma unroll
    for (int m = 0; m < kPerWave; ++m) {
        sum[m] = 0.0f;
#pragma unroll
        for (int n = 0; n < kPerWave; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[m][n][r] = 0.0f;
    }
    const int wm = wave / 2 * kPerWave, wn = wave % 2 * kPerWave;  // the wavefront's first fragments
    Stage s;
    if (begin < end) {
        load(s, begin);
        put(s, 0);
    }
    __syncthreads();
    int buf = 0;
    for (int64_t t0 = begin; t0 < end; t0 += kTokens, buf ^= 1) {
        const bool more = t0 + kTokens < end;
        if (more) load(s, t0 + kTokens);
#pragma unroll
        for (int t = 0; t < kTokens; t += 16) {
            bf16x8 fa[kPerWave], fb[kPerWave];
#pragma unroll
            for (int m = 0; m < kPerWave; ++m) fa[m] = read_fragment(tile_a[buf], wm + m, t, lane);
#pragma unroll
            for (int n = 0; n < kPerWave; ++n) fb[n] = read_fragment(tile_b[buf], wn + n, t, lane);
#pragma unroll
            for (int m = 0; m < kPerWave; ++m) {
#pragma unroll
                for (int n = 0; n < kPerWave; ++n) acc[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[m], fb[n], acc[m][n], 0, 0, 0);
                if constexpr (SUMS)
#pragma unroll
                    for (int i = 0; i < kVec; ++i) sum[m] += (float)fa[m][i];
            }
        }
        if (more) put(s, buf ^ 1);
        __syncthreads();
    }

    // Lane l has column l mod 32 of a fragment's tile, rows 8 (r / 4) + 4 (l / 32) + r mod 4 in register r; a row's sum over the tokens of
    // one half of the lanes each.
    const int64_t gs = (int64_t)split * a.groups + group;
#pragma unroll
    for (int m = 0; m < kPerWave; ++m) {
        if constexpr (SUMS) {
            sum[m] += __shfl_xor(sum[m], 32);
            const int64_t o = o0 + (wm + m) * kFrag + lane;
            if (k0 == 0 && wn == 0 && lane < kFrag && o < a.out) {
                if (a.splits > 1) a.sums[gs * a.out + o] = sum[m];
                else if (a.db.data) finish_sum(a, group, o, sum[m]);
            }
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int in_tile = 8 * (r / 4) + 4 * (lane / 32) + r % 4;
            const int64_t o = o0 + (wm + m) * kFrag + in_tile;
            const float of_row = SUMS ? __shfl(sum[m], in_tile) : 0.0f;
#pragma unroll
            for (int n = 0; n < kPerWave; ++n) {
                const int64_t k = k0 + (wn + n) * kFrag + lane % 32;
                if (o < a.out && k < a.in) {
                    if (a.splits > 1) a.part[(gs * a.out + o) * a.in + k] = acc[m][n][r];
                    else finish(a, group, o, k, acc[m][n][r], of_row);
                }
            }
        }
    }
}

// The splits' parts, added in order.
template <bool SUMS>
__global__ __launch_bounds__(kThreads) void apm_wgrad_join_kernel(WgradArgs a) {
    const int64_t k = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t go = blockIdx.y, group = go / a.out, o = go - group * a.out;
    float sum = 0.0f;
    if constexpr (SUMS)
        for (int s = 0; s < a.splits; ++s) sum += a.sums[((int64_t)s * a.groups + group) * a.out + o];
    if (k < a.in) {
        float v = 0.0f;
        for (int s = 0; s < a.splits; ++s) v += a.part[(((int64_t)s * a.groups + group) * a.out + o) * a.in + k];
        finish(a, group, o, k, v, sum);
    }
    if (SUMS && k == 0 && a.db.data) finish_sum(a, group, o, sum);
}

struct WgradShape {
    int64_t tiles_out, tiles_in, groups;
    int32_t splits;
};
WgradShape wgrad_shape(const apm_weight_grad& w) {
    WgradShape s;
    s.tiles_out = div_up(w.out, kTile), s.tiles_in = div_up(w.in, kTile);
    s.groups = std::max<int64_t>(1, w.n_groups);
    const int64_t tiles = s.tiles_out * s.tiles_in * s.groups;
    s.splits = (int32_t)std::max<int64_t>(1, std::min<int64_t>({512 / tiles, div_up(w.tokens, 4 * kTokens), 64}));
    return s;
}
size_t workspace_of(const apm_weight_grad& w, const WgradShape& s) {
    return s.splits > 1 ? (size_t)s.splits * s.groups * w.out * (w.in + 1) * sizeof(float) : 0;
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
    a.format = w.kept.format, a.dw_type = w.dw.dtype, a.accumulate = w.accumulate;
    const int64_t tiles = s.tiles_out * s.tiles_in, most = max_workgroups(kThreads);
    if (tiles > most / s.splits) return fail(APM_EINVAL, "dw is too large for one product");
    a.tiles = (int32_t)tiles;
    const bool sums = w.bias.data || w.db.data;
    const hipStream_t st = (hipStream_t)stream;
    const int64_t groups_per_launch = most / (tiles * s.splits);
    for (int64_t g = 0; g < s.groups; g += groups_per_launch) {
        a.first_group = (int32_t)g;
        const dim3 grid((unsigned)(tiles * s.splits * std::min(groups_per_launch, s.groups - g)));
        if (sums) hipLaunchKernelGGL(apm_wgrad_kernel<true>, grid, dim3(kThreads), 0, st, a);
        else hipLaunchKernelGGL(apm_wgrad_kernel<false>, grid, dim3(kThreads), 0, st, a);
        APM_HIP(hipGetLastError());
    }
    if (s.splits > 1) {  // so that there are few tiles, and few rows of dw
        const dim3 grid((unsigned)div_up(w.in, kThreads), (unsigned)(s.groups * w.out));
        if (sums) hipLaunchKernelGGL(apm_wgrad_join_kernel<true>, grid, dim3(kThreads), 0, st, a);
        else hipLaunchKernelGGL(apm_wgrad_join_kernel<false>, grid, dim3(kThreads), 0, st, a);
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
