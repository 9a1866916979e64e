// Dropout whose mask is a function of the element's place: y = residual + (u < T ? 0 : x scale), u 16 bits of a counter-based generator, so that nothing is
// stored between the forward and the backward pass.  A counter for each eight columns of a row: its four words are their sixteen-bit numbers.
// HBM-bound: 16384 x 2048 bf16 with a residual 32 us = 6.3 TB/s; the generator's twenty 64-bit products and their mixing for eight elements hide behind that.  All
// accesses are non-temporal (36 us without); one row a wavefront 33.7, four 34.4 when two took 33.0.
#include <algorithm>
#include <cmath>

#include "apm_tok.h"

namespace apm {
namespace {

constexpr int kWave = 64, kThreads = 256, kWaves = kThreads / kWave;
constexpr int kSlice = kWave * kVec;  // columns of a wavefront
constexpr int kRows = 2;     // rows of a wavefront, whose loads are under way together

struct DropoutArgs {
    apm_matrix x, residual, y;
    const uint64_t* seed_at;
    uint64_t seed;
    uint64_t first_row;
    int64_t first, end;  // rows of this launch
    uint32_t slices;
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
    const int lane = (int)threadIdx.x % kWave;
    const uint32_t item = blockIdx.x * kWaves + (uint32_t)__builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), nth = item / a.slices;
    const int64_t r0 = a.first + (int64_t)nth * kRows;
    if (r0 >= a.end) return;
    LaneCols l;
    l.set((int)(item - nth * a.slices) * kSlice + lane * kVec, a.cols);
    Raw<X> x[kRows];
    Raw<Y> residual[kRows];
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
        load_row(x[u], a.x, r0 + u, a.cols, r0 + u < a.end, l);
        if constexpr (RESIDUAL) load_row(residual[u], a.residual, r0 + u, a.cols, r0 + u < a.end, l);
    }
    const uint64_t seed = a.seed + (a.seed_at ? *a.seed_at : 0);
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
        const Philox random((uint32_t)l.col / kVec, a.first_row + (uint64_t)(r0 + u), a.layer, seed);
        settle(x[u], l, a.cols);
        if constexpr (RESIDUAL) settle(residual[u], l, a.cols);
        float v[kVec];
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            v[i] = random[i] < a.bound ? 0.0f : x[u][i] * a.scale;
            if constexpr (RESIDUAL) v[i] += residual[u][i];
        }
        store_row<Y>(a.y, r0 + u, a.cols, r0 + u < a.end, l, v);
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
    for (const apm_matrix& m : {d.x, d.residual})
        if (m.data == d.y.data && (m.dtype != d.y.dtype || (m.stride != d.y.stride && d.rows > 1))) return fail(APM_EINVAL, "y is where x or the residual is, in another form");
    DropoutArgs a{};
    a.x = d.x, a.residual = d.residual, a.y = d.y;
    a.seed_at = d.seed_at, a.seed = d.seed, a.layer = d.layer, a.first_row = (uint64_t)d.first_row;
    a.cols = (int32_t)d.cols, a.slices = (uint32_t)div_up(d.cols, kSlice);
    a.bound = (uint32_t)std::llround(d.p * 65536.0);
    a.scale = a.bound < 65536 ? (float)(65536.0 / (65536.0 - a.bound)) : 0.0f;
    const int64_t most = std::max<int64_t>(1, workgroups_of_launch(kThreads) * kWaves / a.slices) * kRows;  // rows of a launch
    for (a.first = 0; a.first < d.rows; a.first = a.end) {
        a.end = std::min(d.rows, a.first + most);  // the last workgroup can have wavefronts to spare, whose rows are the next launch's: in place they would be dropped out twice
        const dim3 grid((unsigned)div_up(div_up(a.end - a.first, kRows) * a.slices, kWaves)), block(kThreads);
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
