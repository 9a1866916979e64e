// A matrix into 8 bits with a scale for each 32 channels, and back.  HBM-bound: 3 B/element and a byte per block for bf16, 5 for fp32.
#include <algorithm>

#include "apm_act.h"

namespace apm {

// Rows times the distance between them stays in an address.
static bool far_rows(int64_t rows, int64_t stride) { return rows > 1 && stride > ((int64_t)1 << 56) / rows; }

int check_matrix(const char* name, const apm_matrix& m, int64_t rows, int64_t cols, bool written) {
    if (rows == 0) return APM_OK;
    if (!m.data) return fail(APM_EINVAL, "%s is missing", name);
    if (m.dtype != APM_F32 && m.dtype != APM_BF16) return fail(APM_EINVAL, "%s: bad dtype %d", name, m.dtype);
    if ((uintptr_t)m.data % (m.dtype == APM_F32 ? 4 : 2) != 0) return fail(APM_EINVAL, "%s is not aligned to its elements", name);
    if (m.stride < 0 || far_rows(rows, m.stride) || (written && rows > 1 && m.stride < cols))
        return fail(APM_EINVAL, "%s: a row stride of %lld for %lld columns", name, (long long)m.stride, (long long)cols);
    return APM_OK;
}

int check_vector(const char* name, const apm_vector& v) {
    if (!v.data) return APM_OK;
    if (v.dtype != APM_F32 && v.dtype != APM_BF16) return fail(APM_EINVAL, "%s: bad dtype %d", name, v.dtype);
    if ((uintptr_t)v.data % (v.dtype == APM_F32 ? 4 : 2) != 0) return fail(APM_EINVAL, "%s is not aligned to its elements", name);
    return APM_OK;
}

int check_ckpt(const char* name, const apm_ckpt& c, int64_t rows, int64_t cols, bool written) {
    if (rows == 0) return APM_OK;
    if (!c.q || !c.scale) return fail(APM_EINVAL, "%s is missing", name);
    if (c.format != APM_CKPT_I8 && c.format != APM_CKPT_F8) return fail(APM_EINVAL, "%s: bad format %d", name, c.format);
    const int64_t nb = div_up(cols, APM_CKPT_BLOCK);
    if (c.q_stride < 0 || c.scale_stride < 0 || far_rows(rows, c.q_stride) || far_rows(rows, c.scale_stride) || (written && rows > 1 && (c.q_stride < cols || c.scale_stride < nb)))
        return fail(APM_EINVAL, "%s: row strides of %lld and %lld for %lld columns", name, (long long)c.q_stride, (long long)c.scale_stride,
                    (long long)cols);
    return APM_OK;
}

namespace {

// Loads are non-temporal where rows are aligned to them, stores of bf16 and bytes always: what a wavefront of fp32 stores with one
// instruction are halves of cache lines, which then meet in memory.  16384 x 8192 bf16 into 8 bits 63-66 us = 6.2-6.4 TB/s, with the default policy 72;
// 8192 x 20480 back 80 us = 6.3 TB/s, and 85; 8192 x 8192 back to fp32 102 us with non-temporal stores, 62 without; 16384 x 1001 into 8 bits 12.4 us with
// non-temporal loads, 10.7 without.
constexpr int kThreads = 256, kUnroll = 2;
constexpr int kGroupBlocks = kThreads * kUnroll / kQuad;  // blocks of the 8-bit form that a workgroup takes

struct CkptArgs {
    char* x;
    char* q;
    uint8_t* scale;
    int64_t x_stride, q_stride, scale_stride;
    int64_t first_row;
    uint32_t rows, cols, blocks;  // blocks: of a row
    float inv_blocks;
    int32_t format;
};

// Where a quad's block lies.  The workgroup's first block is (row0, block0); b blocks on, rows have wrapped a few times at most
// if they are long, and b / blocks is below 2^8 in any case, so that one correction makes up for the reciprocal's rounding.
struct Place {
    int64_t row;
    int col, n;  // the lane's first column, and how many of its eight exist (0 or less: none)
    uint32_t block;
};
__device__ __forceinline__ Place place_of(const CkptArgs& a, uint32_t row0, uint32_t block0, uint32_t b, int lane_in_quad) {
    const uint32_t at = block0 + b;
    uint32_t r = (uint32_t)((float)at * a.inv_blocks);
    int32_t left = (int32_t)(at - r * a.blocks);
    if (left < 0) r -= 1, left += (int32_t)a.blocks;
    else if (left >= (int32_t)a.blocks) r += 1, left -= (int32_t)a.blocks;
    Place p;
    p.row = (int64_t)row0 + r;
    p.block = (uint32_t)left;
    p.col = left * APM_CKPT_BLOCK + lane_in_quad * kVec;
    p.n = p.row < (int64_t)a.rows ? (int)min((int64_t)kVec, (int64_t)a.cols - p.col) : 0;
    p.row += a.first_row;
    return p;
}

template <class T, bool ALIGNED>
__global__ __launch_bounds__(kThreads) void apm_ckpt_write_kernel(CkptArgs a) {
    const uint32_t first = blockIdx.x * kGroupBlocks, row0 = first / a.blocks, block0 = first - row0 * a.blocks;
    const int in_quad = (int)threadIdx.x % kQuad;
    Place p[kUnroll];
    Raw<T> x[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        p[u] = place_of(a, row0, block0, (uint32_t)(u * (kThreads / kQuad)) + threadIdx.x / kQuad, in_quad);
        x[u].template load<ALIGNED>(a.x + p[u].row * a.x_stride * (int64_t)sizeof(T), p[u].col, p[u].n);
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        float v[kVec];
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = x[u][i];
        uint32_t s;
        const u32x2 w = encode8(v, a.format, &s);
        store_q<true>(a.q + p[u].row * a.q_stride, p[u].col, p[u].n, w);
        if (in_quad == 0 && p[u].n > 0) a.scale[p[u].row * a.scale_stride + p[u].block] = (uint8_t)s;
    }
}

template <class T, bool ALIGNED>
__global__ __launch_bounds__(kThreads) void apm_ckpt_read_kernel(CkptArgs a) {
    const uint32_t first = blockIdx.x * kGroupBlocks, row0 = first / a.blocks, block0 = first - row0 * a.blocks;
    const int in_quad = (int)threadIdx.x % kQuad;
    Place p[kUnroll];
    u32x2 w[kUnroll];
    uint32_t s[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        p[u] = place_of(a, row0, block0, (uint32_t)(u * (kThreads / kQuad)) + threadIdx.x / kQuad, in_quad);
        w[u] = load_q<ALIGNED>(a.q + p[u].row * a.q_stride, p[u].col, p[u].n);
        s[u] = p[u].n > 0 ? a.scale[p[u].row * a.scale_stride + p[u].block] : 0u;
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        float v[kVec];
        decode8(w[u], scale_of(s[u], a.format), a.format, v);
        store8<T, sizeof(T) == sizeof(bf16)>(a.x + p[u].row * a.x_stride * (int64_t)sizeof(T), p[u].col, p[u].n, v);
    }
}

int convert(int64_t rows, int64_t cols, const apm_matrix* x, const apm_ckpt* c, bool to_8, void* stream) {
    if (!x || !c) return fail(APM_EINVAL, "missing argument");
    if (rows < 0 || cols < 1 || cols > INT32_MAX - APM_CKPT_BLOCK) return fail(APM_EINVAL, "bad size %lld x %lld", (long long)rows, (long long)cols);
    int rc = check_matrix("x", *x, rows, cols, !to_8);
    if (rc == APM_OK) rc = check_ckpt("the 8-bit matrix", *c, rows, cols, to_8);
    if (rc != APM_OK || rows == 0) return rc;
    CkptArgs a{};
    a.x = (char*)x->data, a.q = (char*)c->q, a.scale = (uint8_t*)c->scale;
    a.x_stride = x->stride, a.q_stride = c->q_stride, a.scale_stride = c->scale_stride;
    a.cols = (uint32_t)cols, a.blocks = (uint32_t)div_up(cols, APM_CKPT_BLOCK);
    a.inv_blocks = 1.0f / (float)a.blocks;
    a.format = c->format;
    const int64_t size = x->dtype == APM_F32 ? 4 : 2;  // what is loaded: vectors of x, or eight bytes
    const bool aligned = to_8 ? (uintptr_t)x->data % 16 == 0 && x->stride * size % 16 == 0 : (uintptr_t)c->q % 8 == 0 && c->q_stride % 8 == 0;
    const int64_t most = std::max<int64_t>(1, ((int64_t)1 << 30) / a.blocks);  // rows of a launch: block numbers stay in 32 bits
    for (a.first_row = 0; a.first_row < rows; a.first_row += most) {
        a.rows = (uint32_t)std::min(most, rows - a.first_row);
        const dim3 grid((unsigned)div_up((int64_t)a.rows * a.blocks, kGroupBlocks)), block(kThreads);
        const hipStream_t s = (hipStream_t)stream;
        auto start = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, s, a); };
        if (to_8) {
            if (x->dtype == APM_F32) aligned ? start(apm_ckpt_write_kernel<float, true>) : start(apm_ckpt_write_kernel<float, false>);
            else aligned ? start(apm_ckpt_write_kernel<bf16, true>) : start(apm_ckpt_write_kernel<bf16, false>);
        } else {
            if (x->dtype == APM_F32) aligned ? start(apm_ckpt_read_kernel<float, true>) : start(apm_ckpt_read_kernel<float, false>);
            else aligned ? start(apm_ckpt_read_kernel<bf16, true>) : start(apm_ckpt_read_kernel<bf16, false>);
        }
        APM_HIP(hipGetLastError());
    }
    return APM_OK;
}

}  // namespace
}  // namespace apm

extern "C" int apm_ckpt_write(int64_t rows, int64_t cols, const apm_matrix* x, const apm_ckpt* c, void* stream) {
    return apm::guarded([&]() -> int { return apm::convert(rows, cols, x, c, true, stream); });
}

extern "C" int apm_ckpt_read(int64_t rows, int64_t cols, const apm_ckpt* c, const apm_matrix* x, void* stream) {
    return apm::guarded([&]() -> int { return apm::convert(rows, cols, x, c, false, stream); });
}
