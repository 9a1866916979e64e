// Dropout whose mask is a function of the element's place: y = residual + (u < T ? 0 : x scale), u 16 bits of a counter-based generator, so that nothing is
// stored between the forward and the backward pass.  A counter for each eight columns of a row: its four words are their sixteen-bit numbers.
#include <algorithm>
#include <cmath>

#include "apm_tok.h"

namespace apm {
namespace {

constexpr int kThreads = 256, kUnroll = 2;

struct DropoutArgs {
    const char* x;
    const char* residual;
    char* y;
    const uint64_t* seed_at;
    uint64_t seed;
    int64_t x_stride, residual_stride, y_stride;
    int64_t first_row;  // of the launch
    uint64_t counter;   // of that row
    uint32_t rows, vecs;
    float inv_vecs;
    int32_t cols;
    uint32_t bound, layer;
    float scale;
};

// Philox4x32 of ten rounds: two products of 32 x 32 bits a round, of which the low halves become words and the high halves are mixed with the others and
// the key, which goes on by two constants.
struct Philox {
    uint32_t c[4];
    __device__ __forceinline__ Philox(uint32_t block, uint64_t row, uint32_t layer, uint64_t seed) : c{block, (uint32_t)row, (uint32_t)(row >> 32), layer} {
        uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
        for (int i = 0; i < 10; ++i) {
            const uint64_t a = (uint64_t)c[0] * 0xD2511F53u, b = (uint64_t)c[2] * 0xCD9E8D57u;
            c[0] = (uint32_t)(b >> 32) ^ c[1] ^ k0;
            c[2] = (uint32_t)(a >> 32) ^ c[3] ^ k1;
            c[1] = (uint32_t)b, c[3] = (uint32_t)a;
            k0 += 0x9E3779B9u, k1 += 0xBB67AE85u;
        }
    }
    __device__ __forceinline__ uint32_t operator[](int i) const { return (i & 1) ? c[i / 2] >> 16 : c[i / 2] & 0xffffu; }
};

template <class X, class Y, bool RESIDUAL>
__global__ __launch_bounds__(kThreads) void apm_dropout_kernel(DropoutArgs a) {
    const uint32_t first = blockIdx.x * (uint32_t)(kThreads * kUnroll), row0 = first / a.vecs, vec0 = first - row0 * a.vecs;
    const uint64_t seed = a.seed + (a.seed_at ? *a.seed_at : 0);
    Raw<X> x[kUnroll];
    Raw<Y> residual[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        const VecPlace p(row0, vec0, (uint32_t)(u * kThreads) + threadIdx.x, a.vecs, a.inv_vecs, a.cols);
        const int64_t row = a.first_row + p.row;
        const int n = p.row < a.rows ? p.n : 0;
        x[u].load(a.x + row * a.x_stride * (int64_t)sizeof(X), p.col, n);
        if constexpr (RESIDUAL) residual[u].load(a.residual + row * a.residual_stride * (int64_t)sizeof(Y), p.col, n);
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        const VecPlace p(row0, vec0, (uint32_t)(u * kThreads) + threadIdx.x, a.vecs, a.inv_vecs, a.cols);
        const Philox random((uint32_t)p.col / kVec, a.counter + p.row, a.layer, seed);
        float v[kVec];
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            v[i] = random[i] < a.bound ? 0.0f : x[u][i] * a.scale;
            if constexpr (RESIDUAL) v[i] += residual[u][i];
        }
        store8<Y>(a.y + (a.first_row + p.row) * a.y_stride * (int64_t)sizeof(Y), p.col, p.row < a.rows ? p.n : 0, v);
    }
}

int apply(const apm_dropout* dp, void* stream) {
    if (!dp) return fail(APM_EINVAL, "missing argument");
    const apm_dropout& d = *dp;
    if (d.rows < 0 || d.cols < 1 || d.cols > kMostCols || d.first_row < 0) return fail(APM_EINVAL, "bad size %lld x %lld from row %lld", (long long)d.rows, (long long)d.cols, (long long)d.first_row);
    if (!(d.p >= 0.0 && d.p <= 1.0)) return fail(APM_EINVAL, "p = %g is no probability", d.p);
    if (!aligned_to(d.seed_at, 8)) return fail(APM_EINVAL, "seed_at is not aligned to its word");
    int rc = check_matrix("x", d.x, d.rows, d.cols, false);
    if (rc == APM_OK) rc = check_matrix("y", d.y, d.rows, d.cols, true);
    if (rc == APM_OK && d.residual.data) rc = check_matrix("residual", d.residual, d.rows, d.cols, false);
    if (rc != APM_OK || d.rows == 0) return rc;
    if (d.residual.data && d.residual.dtype != d.y.dtype) return fail(APM_EINVAL, "residual and y have different types");
    DropoutArgs a{};
    a.x = (const char*)d.x.data, a.residual = (const char*)d.residual.data, a.y = (char*)d.y.data;
    a.seed_at = d.seed_at, a.seed = d.seed, a.layer = d.layer;
    a.x_stride = d.x.stride, a.residual_stride = d.residual.stride, a.y_stride = d.y.stride;
    a.cols = (int32_t)d.cols, a.vecs = (uint32_t)div_up(d.cols, kVec), a.inv_vecs = 1.0f / (float)a.vecs;
    a.bound = (uint32_t)std::llround(d.p * 65536.0);
    a.scale = a.bound < 65536 ? (float)(65536.0 / (65536.0 - a.bound)) : 0.0f;
    const int64_t most = std::max<int64_t>(1, kMostVecs / a.vecs);
    for (a.first_row = 0; a.first_row < d.rows; a.first_row += most) {
        a.rows = (uint32_t)std::min(most, d.rows - a.first_row);
        a.counter = (uint64_t)d.first_row + (uint64_t)a.first_row;
        const dim3 grid((unsigned)div_up((int64_t)a.rows * a.vecs, kThreads * kUnroll)), block(kThreads);
        const hipStream_t s = (hipStream_t)stream;
        auto start = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, s, a); };
        auto with = [&](auto x, auto y) {
            typedef decltype(x) X;
            typedef decltype(y) Y;
            d.residual.data ? start(apm_dropout_kernel<X, Y, true>) : start(apm_dropout_kernel<X, Y, false>);
        };
        if (d.x.dtype == APM_F32) d.y.dtype == APM_F32 ? with(float(), float()) : with(float(), bf16());
        else d.y.dtype == APM_F32 ? with(bf16(), float()) : with(bf16(), bf16());
        APM_HIP(hipGetLastError());
    }
    return APM_OK;
}

}  // namespace
}  // namespace apm

extern "C" int apm_dropout_apply(const apm_dropout* d, void* stream) {
    return apm::guarded([&]() -> int { return apm::apply(d, stream); });
}
