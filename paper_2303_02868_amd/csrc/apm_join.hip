// Where one block of a residual network ends and the next begins: y = scale x + gate post(branch), n = pre(y), with both
// normalised tensors kept in 8 bits, and the gradients out of those.  HBM-bound in both directions (bf16: 10 B/element
// and the scales, forward x, branch, y, n and two bytes, backward dy, dn, two bytes, dx, dbranch), so a row is read once
// and stays in registers between its sums, held by one wavefront or by as many as it takes.
#include <algorithm>
#include <type_traits>

#include "apm_act.h"

namespace apm {
namespace {

constexpr int kWave = 64, kMaxWaves = 16, kMaxThreads = kWave * kMaxWaves;
static_assert(kMaxThreads * kVec * 2 == APM_JOIN_MAX_COLS, "a row fits the largest workgroup with two vectors a lane");

struct JoinArgs {
    apm_norm_join j;
    float scale, eps_pre, eps_post, inv_cols;
    int64_t first_row;  // of the launch
};

// Sums over the lanes that hold a row.  With several wavefronts through `slots`: kMaxWaves floats for each sum, those of wavefronts that the row does
// not have zero; they may be written again after the next barrier.
template <bool WAVE, int N>
__device__ __forceinline__ void team_sums(float (&x)[N], float* slots, int wave) {
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = wave_sum(x[k]);
    if constexpr (!WAVE) {
        if (threadIdx.x % kWave == 0)
#pragma unroll
            for (int k = 0; k < N; ++k) slots[k * kMaxWaves + wave] = x[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] = row_sum16(slots[k * kMaxWaves + threadIdx.x % kMaxWaves]);
    }
}

// Eight columns of a vector of parameters (`none` where it is absent), or of the gate: loaded, and looked at later, so that several are under way.
struct Param {
    RowAny raw;
    __device__ __forceinline__ void load(const apm_vector& p, int64_t cols, const LaneCols& l) {
        if (p.data) raw.load(p.data, 0, p.dtype, cols, true, l);
    }
    __device__ __forceinline__ void get(const apm_vector& p, int64_t cols, const LaneCols& l, float (&v)[kVec], float none) {
        if (p.data) {
            raw.get(p.dtype, cols, l, v);
        } else {
#pragma unroll
            for (int i = 0; i < kVec; ++i) v[i] = none;
        }
    }
    // A column's gate for all rows, or this row's
    __device__ __forceinline__ void load_gate(const apm_norm_join& j, int64_t row, bool there, const LaneCols& l) {
        raw.load(j.gate.data, j.gate_kind == APM_GATE_FULL ? row * j.gate.stride : 0, j.gate.dtype, j.cols, there, l);
    }
    __device__ __forceinline__ void get_gate(const apm_norm_join& j, const LaneCols& l, float (&g)[kVec]) { raw.get(j.gate.dtype, j.cols, l, g); }
};
// A gate that is one value of a row, likewise
struct Token {
    uint32_t raw;
    __device__ __forceinline__ void load(const apm_norm_join& j, int64_t row, bool there) {
        raw = 0u;
        if (j.gate_kind == APM_GATE_TOKEN && there) raw = j.gate.dtype == APM_F32 ? ((const uint32_t*)j.gate.data)[row * j.gate.stride] : ((const uint16_t*)j.gate.data)[row * j.gate.stride];
    }
    __device__ __forceinline__ float get(const apm_norm_join& j) const {
        return j.gate_kind != APM_GATE_TOKEN ? 1.0f : __builtin_bit_cast(float, j.gate.dtype == APM_F32 ? raw : raw << 16);
    }
};

// z becomes hat(z); elements beyond the row's end are zero before and after.
template <bool WAVE, int VECS>
__device__ __forceinline__ float normalise(float (&z)[VECS][kVec], const LaneCols (&l)[VECS], int32_t kind, float eps, float inv_cols, float* slots) {
    if (kind == APM_NORM_NONE) return 1.0f;
    const int wave = (int)threadIdx.x / kWave;
    if (kind == APM_NORM_LAYER) {
        float s[1] = {0.0f};
#pragma unroll
        for (int v = 0; v < VECS; ++v)
#pragma unroll
            for (int i = 0; i < kVec; ++i) s[0] += z[v][i];
        team_sums<WAVE>(s, slots, wave);
        const float mean = s[0] * inv_cols;
#pragma unroll
        for (int v = 0; v < VECS; ++v)
#pragma unroll
            for (int i = 0; i < kVec; ++i) z[v][i] = i < l[v].n ? z[v][i] - mean : 0.0f;
    }
    float q[1] = {0.0f};
#pragma unroll
    for (int v = 0; v < VECS; ++v)
#pragma unroll
        for (int i = 0; i < kVec; ++i) q[0] = fmaf(z[v][i], z[v][i], q[0]);
    team_sums<WAVE>(q, slots + kMaxWaves, wave);
    const float r = 1.0f / sqrtf(fmaf(q[0], inv_cols, eps));
#pragma unroll
    for (int v = 0; v < VECS; ++v)
#pragma unroll
        for (int i = 0; i < kVec; ++i) z[v][i] *= r;
    return r;
}

// The forward kernel has other wavefronts to run while one waits: it loads these one after the other, in few registers (8192 x 2048: 34.8 us, with
// a norm's weight, bias and gate under way together 38).
__device__ __forceinline__ void affine(const apm_norm& norm, int64_t cols, const LaneCols& l, const float (&z)[kVec], float (&out)[kVec]) {
    Param p;
    float w[kVec], b[kVec];
    p.load(norm.weight, cols, l);
    p.get(norm.weight, cols, l, w, 1.0f);
    p.load(norm.bias, cols, l);
    p.get(norm.bias, cols, l, b, 0.0f);
#pragma unroll
    for (int i = 0; i < kVec; ++i) out[i] = fmaf(z[i], w[i], b[i]);
}

constexpr int kRowsPerGroup = 4;  // of one wavefront each

// One row a team: a wavefront up to 512 columns, else as many as hold it with eight columns a lane, or from 8192 columns on with 16 (16 all along, us: 8192 x
// 5120 with a fp32 stream 131, with eight 111; 8192 x 2048 37 and 34; 8 x 768 6.9 and 4.7).  5.3 TB/s at 8192 x 5120, 5.0 at 8192 x 2048.
template <class R, class A, int VECS, bool WAVE>
__global__ __launch_bounds__(WAVE ? kWave * kRowsPerGroup : kMaxThreads) void apm_join_forward_kernel(JoinArgs a) {
    __shared__ float slots[WAVE ? 1 : 4 * kMaxWaves];
    const apm_norm_join& j = a.j;
    const int lane = WAVE ? (int)threadIdx.x % kWave : (int)threadIdx.x, lanes = WAVE ? kWave : (int)blockDim.x;
    int64_t row = a.first_row + blockIdx.x;
    if constexpr (WAVE) {
        row = a.first_row + (int64_t)blockIdx.x * kRowsPerGroup + __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
        if (row >= j.rows) return;
    }
    LaneCols l[VECS];
    Raw<R> x[VECS];
    Raw<A> b[VECS];
#pragma unroll
    for (int v = 0; v < VECS; ++v) {
        l[v].set((v * lanes + lane) * kVec, j.cols);
        load_row(x[v], j.x, row, j.cols, true, l[v]);
        load_row(b[v], j.branch, row, j.cols, true, l[v]);
    }
    Token token;
    token.load(j, row, true);
    if constexpr (!WAVE) {
        if (threadIdx.x < 4 * kMaxWaves) slots[threadIdx.x] = 0.0f;
        __syncthreads();
    }
    float y[VECS][kVec];
#pragma unroll
    for (int v = 0; v < VECS; ++v) {
        settle(x[v], l[v], j.cols);
#pragma unroll
        for (int i = 0; i < kVec; ++i) y[v][i] = a.scale * x[v][i];
    }
    if (j.branch.data) {
        float z[VECS][kVec];
#pragma unroll
        for (int v = 0; v < VECS; ++v) {
            settle(b[v], l[v], j.cols);
#pragma unroll
            for (int i = 0; i < kVec; ++i) z[v][i] = b[v][i];
        }
        const float r = normalise<WAVE>(z, l, j.post.kind, a.eps_post, a.inv_cols, slots);
        if (j.post.rstd && lane == 0) j.post.rstd[row] = r;
#pragma unroll
        for (int v = 0; v < VECS; ++v) {
            if (j.post.ckpt.q) keep(j.post.ckpt, row, j.cols, true, l[v], z[v]);
            float c[kVec], g[kVec];
            affine(j.post, j.cols, l[v], z[v], c);
            if (j.gate_kind == APM_GATE_CHANNEL || j.gate_kind == APM_GATE_FULL) {
                Param gate;
                gate.load_gate(j, row, true, l[v]);
                gate.get_gate(j, l[v], g);
            } else {
#pragma unroll
                for (int i = 0; i < kVec; ++i) g[i] = token.get(j);
            }
#pragma unroll
            for (int i = 0; i < kVec; ++i) y[v][i] = i < l[v].n ? fmaf(g[i], c[i], y[v][i]) : 0.0f;
        }
    }
    if (j.y.data) {
#pragma unroll
        for (int v = 0; v < VECS; ++v) store_row<R>(j.y, row, j.cols, true, l[v], y[v]);
    }
    if (!j.n.data && !j.pre.ckpt.q && !j.pre.rstd) return;
    const float r = normalise<WAVE>(y, l, j.pre.kind, a.eps_pre, a.inv_cols, slots + (WAVE ? 0 : 2 * kMaxWaves));
    if (j.pre.rstd && lane == 0) j.pre.rstd[row] = r;
#pragma unroll
    for (int v = 0; v < VECS; ++v) {
        if (j.pre.ckpt.q) keep(j.pre.ckpt, row, j.cols, true, l[v], y[v]);
        if (j.n.data) {
            float o[kVec];
            affine(j.pre, j.cols, l[v], y[v], o);
            store_row<A>(j.n, row, j.cols, true, l[v], o);
        }
    }
}

// ---- backward -----------------------------------------------------------------------------------
// Sums over rows: every thread adds up its columns of its team's rows in LDS, where nobody else touches them, the teams of a workgroup
// are added at the end, and the workgroups' sums, which lie in the workspace, by a second kernel, all in one order.
// Per column: dn hat1, dn, and D hat2, D (times the gate, unless it has one value for the column, which then enters at the end).
enum { kDnHat, kDn, kDHat, kD, kSums };

struct BackArgs {
    apm_norm_join j;
    apm_norm_join_grads g;
    float scale, inv_cols;
    int32_t waves, teams;  // wavefronts of a team, teams of a workgroup
    float* part;           // [workgroups][kSums][cols]
};

__device__ __forceinline__ void finish_column(const apm_norm_join& j, const apm_norm_join_grads& g, int64_t c, const float (&s)[kSums]) {
    if (g.dpre_weight.data) store1(g.dpre_weight.data, g.dpre_weight.dtype, c, s[kDnHat]);
    if (g.dpre_bias.data) store1(g.dpre_bias.data, g.dpre_bias.dtype, c, s[kDn]);
    float gate = 1.0f;
    if (j.gate_kind == APM_GATE_CHANNEL) {
        gate = load1(j.gate.data, j.gate.dtype, c);
        if (g.dgate.data) {
            const float w = j.post.weight.data ? load1(j.post.weight.data, j.post.weight.dtype, c) : 1.0f;
            const float b = j.post.bias.data ? load1(j.post.bias.data, j.post.bias.dtype, c) * s[kD] : 0.0f;
            store1(g.dgate.data, g.dgate.dtype, c, fmaf(w, s[kDHat], b));
        }
    }
    if (g.dpost_weight.data) store1(g.dpost_weight.data, g.dpost_weight.dtype, c, gate * s[kDHat]);
    if (g.dpost_bias.data) store1(g.dpost_bias.data, g.dpost_bias.dtype, c, gate * s[kD]);
}

// A row's part of a lane, as loaded.
template <class R, class A, int VECS>
struct RowRaw {
    Raw<R> dy[VECS];
    Raw<A> dn[VECS];
    Kept k1[VECS], k2[VECS];
    uint32_t r1, r2;
    Token token;
    __device__ __forceinline__ void load(const BackArgs& a, int64_t row, const LaneCols (&l)[VECS]) {
        const bool there = row < a.j.rows;
        r1 = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(row_buffer(a.j.pre.rstd, row * 4, there ? 4u : 0u), 0, 0, 0);
        r2 = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(row_buffer(a.j.post.rstd, row * 4, there ? 4u : 0u), 0, 0, 0);
        token.load(a.j, row, there);
#pragma unroll
        for (int v = 0; v < VECS; ++v) {
            load_row(dy[v], a.g.dy, row, a.j.cols, there, l[v]);
            load_row(dn[v], a.g.dn, row, a.j.cols, there, l[v]);
            k1[v].load(a.j.pre.ckpt, row, a.j.cols, there, l[v]);
            k2[v].load(a.j.post.ckpt, row, a.j.cols, there, l[v]);
        }
    }
};

// ONE: one workgroup, which also does the second kernel's work (in a variant of its own, as it costs the others up to 0.8 us to have the code).
// COLUMN: the gate has one value for a column, or there is none: it then enters with the norm's weight, and at the end.
// VECS 1: a lane has eight columns, and while a row is worked on the next one's loads are under way, so that the lanes of a CU's 16 wavefronts have two
// rows' worth of loads out.  VECS 2, for rows that 16 wavefronts do not hold otherwise: no registers for either.
// The first row is on its way before the weights are asked for, and they all before one of them is looked at (127 x 10215 in fp32: 54 us, so 42).
// 8192 x 5120 with a fp32 stream: 106 us = 5.5 TB/s; of that 4.6 for the second kernel.
constexpr int kSlotSums = 5;  // two for the first norm, three for the second and the gate
template <class R, class A, int VECS, bool WAVE, bool BIAS, bool COLUMN, bool ONE>
__global__ __launch_bounds__(kMaxThreads) void apm_join_backward_kernel(BackArgs a) {
    // The teams' slots, twice; then the sums, four at a time of a thread's.
    extern __shared__ __attribute__((aligned(16))) float lds[];
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    constexpr bool kAhead = VECS == 1;
    constexpr int kAccs = BIAS ? 4 : 2, kInLds = VECS == 1 ? kAccs : 2;
    const apm_norm_join& j = a.j;
    const int threads = (int)blockDim.x, slots_size = WAVE ? 0 : 2 * a.teams * kSlotSums * kMaxWaves;
    f32x4* const sums = (f32x4*)(lds + slots_size) + threadIdx.x;  // [sum][vector][half][thread]
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const int waves = WAVE ? 1 : a.waves, team = WAVE ? wave : wave / waves, in_team = wave - team * waves;
    const int lanes = waves * kWave, lane = in_team * kWave + (int)threadIdx.x % kWave;
    LaneCols l[VECS];
#pragma unroll
    for (int v = 0; v < VECS; ++v) l[v].set((v * lanes + lane) * kVec, j.cols);
    const int64_t step = (int64_t)gridDim.x * a.teams;
    const int64_t begin = (int64_t)blockIdx.x * a.teams;  // the workgroup's first row: all its wavefronts walk as often
    int64_t row = begin + team;
    RowRaw<R, A, VECS> next;
    if constexpr (kAhead) next.load(a, row, l);
    const bool by_column = COLUMN && j.gate_kind == APM_GATE_CHANNEL;
    float w1[VECS][kVec], w2[VECS][kVec], b2[VECS][kVec];
    // w1 the first norm's weight, w2 the second's times a column's gate, b2 the second's bias
    auto weights = [&](int v, bool first, bool second) {
        Param weight1, weight2, gate, bias2;
        if (first) weight1.load(j.pre.weight, j.cols, l[v]);
        if (second) {
            weight2.load(j.post.weight, j.cols, l[v]);
            if (by_column) gate.load_gate(j, 0, true, l[v]);
            if (!COLUMN) bias2.load(j.post.bias, j.cols, l[v]);
        }
        if (first) weight1.get(j.pre.weight, j.cols, l[v], w1[v], 1.0f);
        if (second) {
            weight2.get(j.post.weight, j.cols, l[v], w2[v], 1.0f);
            if (by_column) {
                float g[kVec];
                gate.get_gate(j, l[v], g);
#pragma unroll
                for (int i = 0; i < kVec; ++i) w2[v][i] *= g[i];
            }
#pragma unroll
            for (int i = 0; i < kVec; ++i) w2[v][i] = i < l[v].n ? w2[v][i] : 0.0f;  // what is no column adds nothing to the second norm's sums
            if (!COLUMN) bias2.get(j.post.bias, j.cols, l[v], b2[v], 0.0f);
        }
    };
    if constexpr (kAhead) weights(0, true, true);
    if constexpr (!WAVE) {
        for (int i = (int)threadIdx.x; i < slots_size; i += threads) lds[i] = 0.0f;
        __syncthreads();
    }
#pragma unroll
    for (int k = 0; k < kInLds * VECS * 2; ++k) sums[k * threads] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    float more[kAccs > kInLds ? kAccs - kInLds : 1][VECS][kVec] = {};  // where LDS does not hold all
    auto add = [&](int k, int v, const float (&x)[kVec], const float (&y)[kVec]) {  // sum k += x y
        if (k < kInLds) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                f32x4 s = sums[((k * VECS + v) * 2 + h) * threads];
#pragma unroll
                for (int i = 0; i < 4; ++i) s[i] = fmaf(x[4 * h + i], y[4 * h + i], s[i]);
                sums[((k * VECS + v) * 2 + h) * threads] = s;
            }
        } else {
#pragma unroll
            for (int i = 0; i < kVec; ++i) more[k < kInLds ? 0 : k - kInLds][v][i] = fmaf(x[i], y[i], more[k < kInLds ? 0 : k - kInLds][v][i]);
        }
    };
    float ones[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) ones[i] = 1.0f;
    const bool through1 = j.pre.kind != APM_NORM_NONE, through2 = a.g.dbranch.data && j.post.kind != APM_NORM_NONE;
    const bool mean1 = j.pre.kind == APM_NORM_LAYER, mean2 = through2 && j.post.kind == APM_NORM_LAYER;
    int turn = 0;
    for (int64_t at = begin; at < j.rows; at += step, row += step, turn ^= 1) {
        if constexpr (!kAhead) next.load(a, row, l);
        RowRaw<R, A, VECS> cur = next;
#pragma unroll
        for (int v = 0; v < VECS; ++v) {
            settle(cur.dy[v], l[v], j.cols);
            settle(cur.dn[v], l[v], j.cols);
            cur.k1[v].settle(l[v], j.cols);
            cur.k2[v].settle(l[v], j.cols);
        }
        const bool there = row < j.rows;
        const float r1 = __builtin_bit_cast(float, cur.r1), r2 = __builtin_bit_cast(float, cur.r2);
        const float token = cur.token.get(j);
        if constexpr (kAhead) next.load(a, row + step, l);
        float* slots = lds + (turn * a.teams + team) * kSlotSums * kMaxWaves;
        float D[VECS][kVec];
        {
            float z[VECS][kVec], s[2] = {0.0f, 0.0f};
#pragma unroll
            for (int v = 0; v < VECS; ++v) {
                cur.k1[v].get(j.pre.ckpt.format, z[v]);
                if constexpr (!kAhead) weights(v, true, false);
                float dn[kVec];
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    dn[i] = cur.dn[v][i];
                    D[v][i] = dn[i] * w1[v][i];
                    s[0] = fmaf(D[v][i], z[v][i], s[0]);
                }
                add(0, v, dn, z[v]);
                if constexpr (BIAS) add(2, v, dn, ones);
            }
            if (through1) {
                if (mean1) {
#pragma unroll
                    for (int v = 0; v < VECS; ++v)
#pragma unroll
                        for (int i = 0; i < kVec; ++i) s[1] += D[v][i];
                    team_sums<WAVE>(s, slots, in_team);
                } else {
                    float one[1] = {s[0]};
                    team_sums<WAVE>(one, slots, in_team);
                    s[0] = one[0];
                }
                const float k = s[0] * a.inv_cols, m = s[1] * a.inv_cols;
#pragma unroll
                for (int v = 0; v < VECS; ++v)
#pragma unroll
                    for (int i = 0; i < kVec; ++i) D[v][i] = r1 * (D[v][i] - fmaf(z[v][i], k, m));
            }
        }
        if (!there) {  // a team without a row adds nothing to the sums, also where a weight is infinite
#pragma unroll
            for (int v = 0; v < VECS; ++v)
#pragma unroll
                for (int i = 0; i < kVec; ++i) D[v][i] = 0.0f;
        }
#pragma unroll
        for (int v = 0; v < VECS; ++v) {
            float o[kVec];
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                D[v][i] += cur.dy[v][i];
                o[i] = a.scale * D[v][i];
            }
            store_row<R>(a.g.dx, row, j.cols, there, l[v], o);
        }
        {
            float z[VECS][kVec], s[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int v = 0; v < VECS; ++v) {
                cur.k2[v].get(j.post.ckpt.format, z[v]);
                if constexpr (!kAhead) weights(v, false, true);
                if constexpr (!COLUMN) {
                    if (a.g.dgate.data) {
                        float o[kVec];
#pragma unroll
                        for (int i = 0; i < kVec; ++i) {
                            o[i] = D[v][i] * fmaf(z[v][i], w2[v][i], b2[v][i]);
                            s[2] += o[i];
                        }
                        if (j.gate_kind == APM_GATE_FULL) {
                            if (a.g.dgate.dtype == APM_F32) store_row<float>(a.g.dgate, row, j.cols, there, l[v], o);
                            else store_row<bf16>(a.g.dgate, row, j.cols, there, l[v], o);
                        }
                    }
                    float g[kVec];
                    if (j.gate_kind == APM_GATE_FULL) {
                        Param gate;
                        gate.load_gate(j, row, there, l[v]);
                        gate.get_gate(j, l[v], g);
                    } else {
#pragma unroll
                        for (int i = 0; i < kVec; ++i) g[i] = token;
                    }
#pragma unroll
                    for (int i = 0; i < kVec; ++i) D[v][i] *= g[i];
                }
                add(1, v, D[v], z[v]);
                if constexpr (BIAS) add(3, v, D[v], ones);
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    D[v][i] *= w2[v][i];
                    s[0] = fmaf(D[v][i], z[v][i], s[0]);
                }
                if (mean2) {
#pragma unroll
                    for (int i = 0; i < kVec; ++i) s[1] += D[v][i];
                }
            }
            if (!COLUMN || mean2) {
                team_sums<WAVE>(s, slots + 2 * kMaxWaves, in_team);
                if (!COLUMN && j.gate_kind == APM_GATE_TOKEN && a.g.dgate.data && lane == 0 && there)
                    store1(a.g.dgate.data, a.g.dgate.dtype, row * a.g.dgate.stride, s[2]);
            } else if (through2) {
                float one[1] = {s[0]};
                team_sums<WAVE>(one, slots + 2 * kMaxWaves, in_team);
                s[0] = one[0];
            }
            const float k = s[0] * a.inv_cols, m = mean2 ? s[1] * a.inv_cols : 0.0f;
#pragma unroll
            for (int v = 0; v < VECS; ++v) {
                float o[kVec];
#pragma unroll
                for (int i = 0; i < kVec; ++i) o[i] = r2 * (D[v][i] - fmaf(z[v][i], k, m));
                if (!through2) {  // without a norm hat2, which may be NaN, has no part in it
#pragma unroll
                    for (int i = 0; i < kVec; ++i) o[i] = D[v][i];
                }
                store_row<A>(a.g.dbranch, row, j.cols, there, l[v], o);
            }
        }
    }
    // The teams' sums of four columns, the `half`-th four of vector `vec` of the row
    constexpr int kIndex[4] = {kDnHat, kDHat, kDn, kD};
    auto four = [&](int at, int half, int vec) {
        const int v = VECS == 1 ? 0 : vec / lanes;
        const f32x4* p = (const f32x4*)(lds + slots_size) + ((at * VECS + v) * 2 + half) * threads + vec - v * lanes;
        f32x4 s = p[0];
        for (int m = 1; m < a.teams; ++m) s += p[m * lanes];
        return s;
    };
    const int vectors = ((int)j.cols + kVec - 1) / kVec, fours = 2 * vectors;
    // Four columns a thread, which are next to its neighbours'
    auto store_sums = [&](int first, int count) {
        float* mine = a.part + (int64_t)blockIdx.x * kSums * j.cols;
        for (int at = 0; at < count; ++at) {
            float* to = mine + (int64_t)kIndex[first + at] * j.cols;
            for (int i = (int)threadIdx.x; i < fours; i += threads) {
                const f32x4 s = four(at, i % 2, i / 2);
                const int c = i * 4;
                if (c + 4 <= (int)j.cols) {
                    store_at<false>(__builtin_bit_cast(u32x4, s), (u32x4_any*)(to + c));
                } else {
#pragma unroll
                    for (int e = 0; e < 3; ++e)
                        if (c + e < (int)j.cols) to[c + e] = s[e];
                }
            }
        }
    };
    __syncthreads();
    if constexpr (ONE) {
        for (int c = (int)threadIdx.x; c < (int)j.cols; c += threads) {
            const float* p = lds + slots_size + (c % kVec / 4 * threads + c / kVec) * 4 + c % 4;
            float s[kSums] = {};
            for (int m = 0; m < a.teams; ++m, p += lanes * 4)
#pragma unroll
                for (int k = 0; k < kInLds; ++k) s[kIndex[k]] += p[k * 8 * threads];
            finish_column(j, a.g, c, s);
        }
        return;
    }
    store_sums(0, kInLds);
    if constexpr (kAccs > kInLds) {
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kAccs - kInLds; ++k)
#pragma unroll
            for (int v = 0; v < VECS; ++v)
#pragma unroll
                for (int h = 0; h < 2; ++h) sums[((k * VECS + v) * 2 + h) * threads] = f32x4{more[k][v][4 * h], more[k][v][4 * h + 1], more[k][v][4 * h + 2], more[k][v][4 * h + 3]};
        __syncthreads();
        store_sums(kInLds, kAccs - kInLds);
    }
}

// The workgroups' sums of 32 columns: 32 lanes side by side, 32 parts at a time, eight of them under way.
constexpr int kSide = 32;
template <bool BIAS>
__global__ __launch_bounds__(kSide * kSide) void apm_join_sums_kernel(apm_norm_join j, apm_norm_join_grads g, const float* part, int32_t parts) {
    __shared__ float lds[kSums][kSide][kSide + 1], all[kSums][kSide];
    const int x = (int)threadIdx.x % kSide, y = (int)threadIdx.x / kSide;
    const int64_t c = (int64_t)blockIdx.x * kSide + x;
    float t[kSums] = {};
    if (c < j.cols) {
        for (int32_t p = y; p < parts; p += 8 * kSide) {
            float v[kSums][8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int k = 0; k < kSums; ++k)
                    if (BIAS || k == kDnHat || k == kDHat) v[k][i] = p + i * kSide < parts ? part[((int64_t)(p + i * kSide) * kSums + k) * j.cols + c] : 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int k = 0; k < kSums; ++k)
                    if (BIAS || k == kDnHat || k == kDHat) t[k] += v[k][i];
        }
    }
#pragma unroll
    for (int k = 0; k < kSums; ++k) lds[k][y][x] = t[k];
    __syncthreads();
    if (y < kSums) {
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < kSide; ++i) s += lds[y][i][x];
        all[y][x] = s;
    }
    __syncthreads();
    if (y == 0 && c < j.cols) {
        float s[kSums];
#pragma unroll
        for (int k = 0; k < kSums; ++k) s[k] = all[k][x];
        finish_column(j, g, c, s);
    }
}

// ---- entry points -------------------------------------------------------------------------------

int check_norm(const char* name, const apm_norm& m, int64_t rows, int64_t cols) {
    if (m.kind < APM_NORM_NONE || m.kind > APM_NORM_LAYER) return fail(APM_EINVAL, "%s: bad norm kind %d", name, m.kind);
    if (!(m.eps >= 0.0)) return fail(APM_EINVAL, "%s: eps must not be negative", name);
    int rc = check_vector("a norm's weight", m.weight);
    if (rc == APM_OK) rc = check_vector("a norm's bias", m.bias);
    if (rc == APM_OK && (uintptr_t)m.rstd % 4 != 0) rc = fail(APM_EINVAL, "%s: rstd is not aligned to its elements", name);
    return rc;
}

int check_join(const apm_norm_join& j) {
    if (j.rows < 0 || j.cols < 1 || j.cols > APM_JOIN_MAX_COLS)
        return fail(APM_EINVAL, "bad size %lld x %lld (at most %d columns)", (long long)j.rows, (long long)j.cols, APM_JOIN_MAX_COLS);
    if (j.gate_kind < APM_GATE_NONE || j.gate_kind > APM_GATE_FULL) return fail(APM_EINVAL, "bad gate kind %d", j.gate_kind);
    if (j.gate_kind == APM_GATE_NONE ? j.gate.data != nullptr : !j.gate.data && (j.rows > 0 || j.gate_kind == APM_GATE_CHANNEL)) return fail(APM_EINVAL, "gate and gate_kind contradict each other");
    int rc = check_norm("pre", j.pre, j.rows, j.cols);
    if (rc == APM_OK) rc = check_norm("post", j.post, j.rows, j.cols);
    if (rc == APM_OK && j.gate.data) rc = check_matrix("gate", j.gate, j.gate_kind == APM_GATE_CHANNEL ? 1 : j.rows, j.cols, false);
    return rc;
}

// Types of the residual stream and of what goes in and out of blocks.
int check_types(const apm_matrix& res, const apm_matrix& act) {
    if (res.data && act.data && res.dtype == APM_BF16 && act.dtype == APM_F32)
        return fail(APM_EINVAL, "a bf16 residual stream with fp32 activations is not supported");
    return APM_OK;
}

// Calls go(R(), A()) with the element types.
template <class F>
auto with_types(int32_t res, int32_t act, F&& go) {
    if (res == APM_BF16) return go(bf16(), bf16());
    if (act == APM_BF16) return go(float(), bf16());
    return go(float(), float());
}

int forward(const apm_norm_join* jp, void* stream) {
    if (!jp) return fail(APM_EINVAL, "missing argument");
    const apm_norm_join& j = *jp;
    int rc = check_join(j);
    if (rc != APM_OK) return rc;
    rc = check_matrix("x", j.x, j.rows, j.cols, false);
    if (rc == APM_OK && j.branch.data) rc = check_matrix("branch", j.branch, j.rows, j.cols, false);
    if (rc == APM_OK && j.y.data) rc = check_matrix("y", j.y, j.rows, j.cols, true);
    if (rc == APM_OK && j.n.data) rc = check_matrix("n", j.n, j.rows, j.cols, true);
    if (rc == APM_OK && j.pre.ckpt.q) rc = check_ckpt("pre.ckpt", j.pre.ckpt, j.rows, j.cols, true);
    if (rc == APM_OK && j.post.ckpt.q) rc = check_ckpt("post.ckpt", j.post.ckpt, j.rows, j.cols, true);
    if (rc != APM_OK) return rc;
    if (j.rows > 0 && !j.branch.data && (j.gate.data || j.post.kind != APM_NORM_NONE || j.post.weight.data || j.post.bias.data || j.post.ckpt.q || j.post.rstd))
        return fail(APM_EINVAL, "a gate or a norm after the block, but no branch");
    if (j.y.data && j.y.dtype != j.x.dtype) return fail(APM_EINVAL, "x and y have different types");
    if (j.branch.data && j.n.data && j.branch.dtype != j.n.dtype) return fail(APM_EINVAL, "branch and n have different types");
    const apm_matrix& act = j.branch.data ? j.branch : j.n;
    rc = check_types(j.x, act);
    if (rc != APM_OK || j.rows == 0) return rc;
    JoinArgs a{j, (float)j.residual_scale, (float)j.pre.eps, (float)j.post.eps, (float)(1.0 / (double)j.cols), 0};
    const hipError_t e = with_types(j.x.dtype, act.data ? act.dtype : APM_BF16, [&](auto r, auto t) {
        using R = decltype(r);
        using A = decltype(t);
        const hipStream_t s = (hipStream_t)stream;
        auto start = [&](auto kernel, int64_t rows_per_group, int64_t threads) {
            const int64_t most = max_workgroups((int)threads) * rows_per_group;  // rows of a launch
            for (a.first_row = 0; a.first_row < j.rows; a.first_row += most) {
                const int64_t rows = std::min(most, j.rows - a.first_row);
                hipLaunchKernelGGL(kernel, dim3((unsigned)div_up(rows, rows_per_group)), dim3((unsigned)threads), 0, s, a);
                const hipError_t e = hipGetLastError();
                if (e != hipSuccess) return e;
            }
            return hipSuccess;
        };
        if (j.cols <= kWave * kVec) return start(apm_join_forward_kernel<R, A, 1, true>, kRowsPerGroup, kWave * kRowsPerGroup);
        if (j.cols <= kMaxThreads * kVec) return start(apm_join_forward_kernel<R, A, 1, false>, 1, div_up(j.cols, kWave * kVec) * kWave);
        return start(apm_join_forward_kernel<R, A, 2, false>, 1, div_up(j.cols, kWave * kVec * 2) * kWave);
    });
    APM_HIP(e);
    return APM_OK;
}

// How many workgroups walk the rows, and with how many teams: one workgroup a CU, of as many teams as 16 wavefronts make, so that there are few
// sums of workgroups to add (16384 x 768, us when this was chosen: 50 with 16 wavefronts, 55 with workgroups of 4, of which four share a CU; with
// LayerNorm and biases 42 now), but no more than all CUs have rows for (256 x 768: 14.1 us with as many as there are, 10.5 with one).
constexpr int64_t kCus = 256;
struct BackShape {
    int vecs, waves, teams;
    int64_t groups;
    bool one;  // workgroup, and no second kernel: few rows, whose time is the host's (8 x 768: 16 us, with a second launch 19)
};
BackShape back_shape(int64_t rows, int64_t cols) {
    BackShape b;
    b.vecs = cols <= (int64_t)kMaxThreads * kVec ? 1 : 2;
    b.waves = (int)div_up(cols, kWave * kVec * b.vecs);
    b.teams = kMaxWaves / b.waves;
    b.groups = 1;
    b.one = b.vecs == 1 && rows <= b.teams;
    if (!b.one) {
        b.teams = (int)std::clamp<int64_t>(div_up(rows, kCus), 1, b.teams);
        b.groups = std::clamp<int64_t>(div_up(rows, b.teams), 1, kCus);
    }
    return b;
}

int backward(const apm_norm_join* jp, const apm_norm_join_grads* gp, void* workspace, size_t workspace_bytes, void* stream) {
    if (!jp || !gp) return fail(APM_EINVAL, "missing argument");
    const apm_norm_join& j = *jp;
    const apm_norm_join_grads& g = *gp;
    int rc = check_join(j);
    if (rc != APM_OK) return rc;
    if (j.rows > 0 && !g.dn.data && !g.dy.data) return fail(APM_EINVAL, "neither dn nor dy is given");
    const apm_matrix* m[4] = {&g.dn, &g.dy, &g.dx, &g.dbranch};
    const char* name[4] = {"dn", "dy", "dx", "dbranch"};
    for (int k = 0; k < 4 && rc == APM_OK; ++k)
        if (m[k]->data) rc = check_matrix(name[k], *m[k], j.rows, j.cols, k >= 2);
    const apm_vector* v[4] = {&g.dpre_weight, &g.dpre_bias, &g.dpost_weight, &g.dpost_bias};
    const char* vname[4] = {"dpre_weight", "dpre_bias", "dpost_weight", "dpost_bias"};
    for (int k = 0; k < 4 && rc == APM_OK; ++k) rc = check_vector(vname[k], *v[k]);
    if (rc == APM_OK && g.dgate.data) {
        if (j.gate_kind == APM_GATE_NONE) return fail(APM_EINVAL, "dgate without a gate");
        rc = check_matrix("dgate", g.dgate, j.gate_kind == APM_GATE_CHANNEL ? 1 : j.rows, j.gate_kind == APM_GATE_TOKEN ? 1 : j.cols, true);
    }
    if (rc != APM_OK) return rc;
    if (g.dy.data && g.dx.data && g.dy.dtype != g.dx.dtype) return fail(APM_EINVAL, "dy and dx have different types");
    if (g.dn.data && g.dbranch.data && g.dn.dtype != g.dbranch.dtype) return fail(APM_EINVAL, "dn and dbranch have different types");
    const apm_matrix& res = g.dy.data ? g.dy : g.dx;
    const apm_matrix& act = g.dn.data ? g.dn : g.dbranch;
    rc = check_types(res, act);
    if (rc != APM_OK) return rc;
    const bool need1 = g.dn.data && (j.pre.kind != APM_NORM_NONE || g.dpre_weight.data);
    const bool need2 = g.dgate.data || g.dpost_weight.data || (g.dbranch.data && j.post.kind != APM_NORM_NONE);
    BackArgs a{j, g, (float)j.residual_scale, (float)(1.0 / (double)j.cols), 0, 0, (float*)workspace};
    if (need1) rc = check_ckpt("pre.ckpt", j.pre.ckpt, j.rows, j.cols, false);
    else a.j.pre.ckpt.q = nullptr;
    if (rc == APM_OK && need2) rc = check_ckpt("post.ckpt", j.post.ckpt, j.rows, j.cols, false);
    else a.j.post.ckpt.q = nullptr;
    if (rc != APM_OK) return rc;
    if (j.rows > 0 && g.dn.data && j.pre.kind != APM_NORM_NONE && !j.pre.rstd) return fail(APM_EINVAL, "pre.rstd is missing");
    if (j.rows > 0 && g.dbranch.data && j.post.kind != APM_NORM_NONE && !j.post.rstd) return fail(APM_EINVAL, "post.rstd is missing");
    // What the formulas do not name is not read, and 0 is no factor: a gradient that is missing stays zero beside an infinite weight.
    if (!g.dn.data) a.j.pre.kind = APM_NORM_NONE, a.j.pre.weight.data = nullptr;
    if (a.j.pre.kind == APM_NORM_NONE) a.j.pre.rstd = nullptr;
    if (!g.dbranch.data || j.post.kind == APM_NORM_NONE) a.j.post.rstd = nullptr;
    if (!g.dbranch.data && !g.dgate.data) a.j.post.weight.data = nullptr;
    if (!g.dgate.data) a.j.post.bias.data = nullptr;
    if (workspace_bytes < apm_norm_join_workspace_bytes(j.rows, j.cols)) return fail(APM_ENOMEM, "the workspace is too small");
    if (!workspace || (uintptr_t)workspace % 16 != 0) return fail(APM_EINVAL, "the workspace is missing or not aligned to 16 bytes");
    const BackShape b = back_shape(j.rows, j.cols);
    a.waves = b.waves, a.teams = b.teams;
    const bool bias = g.dpre_bias.data || g.dpost_bias.data || (g.dgate.data && j.gate_kind == APM_GATE_CHANNEL && j.post.bias.data);
    const bool sums = bias || g.dpre_weight.data || g.dpost_weight.data || (g.dgate.data && j.gate_kind == APM_GATE_CHANNEL);
    const hipStream_t s = (hipStream_t)stream;
    const dim3 grid((unsigned)b.groups), block((unsigned)(b.teams * b.waves * kWave));
    const size_t shared = ((size_t)block.x * kVec * b.vecs * (b.vecs == 1 && bias ? 4 : 2) + (b.waves > 1 ? (size_t)2 * b.teams * kSlotSums * kMaxWaves : 0)) * sizeof(float);
    with_types(res.data ? res.dtype : act.data ? act.dtype : APM_BF16, act.data ? act.dtype : APM_BF16, [&](auto r, auto t) {
        using R = decltype(r);
        using A = decltype(t);
        auto start = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, shared, s, a); };
        const bool column = j.gate_kind == APM_GATE_NONE || j.gate_kind == APM_GATE_CHANNEL;
        auto with = [&](auto vecs, auto wave) {
            constexpr int V = decltype(vecs)::value;
            constexpr bool W = decltype(wave)::value;
            auto go = [&](auto alone) {
                constexpr bool O = decltype(alone)::value;
                if (column) bias ? start(apm_join_backward_kernel<R, A, V, W, true, true, O>) : start(apm_join_backward_kernel<R, A, V, W, false, true, O>);
                else bias ? start(apm_join_backward_kernel<R, A, V, W, true, false, O>) : start(apm_join_backward_kernel<R, A, V, W, false, false, O>);
            };
            if constexpr (V == 1) {
                if (b.one) return go(std::true_type());
            }
            go(std::false_type());
        };
        if (b.waves == 1) with(std::integral_constant<int, 1>(), std::true_type());
        else if (b.vecs == 1) with(std::integral_constant<int, 1>(), std::false_type());
        else with(std::integral_constant<int, 2>(), std::false_type());
    });
    APM_HIP(hipGetLastError());
    if (sums && !b.one) {
        const dim3 parts((unsigned)div_up(j.cols, kSide)), all(kSide * kSide);
        if (bias) hipLaunchKernelGGL(apm_join_sums_kernel<true>, parts, all, 0, s, j, g, a.part, (int32_t)b.groups);
        else hipLaunchKernelGGL(apm_join_sums_kernel<false>, parts, all, 0, s, j, g, a.part, (int32_t)b.groups);
        APM_HIP(hipGetLastError());
    }
    return APM_OK;
}

}  // namespace
}  // namespace apm

extern "C" int apm_norm_join_forward(const apm_norm_join* j, void* stream) {
    return apm::guarded([&]() -> int { return apm::forward(j, stream); });
}

extern "C" size_t apm_norm_join_workspace_bytes(int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 1 || cols > APM_JOIN_MAX_COLS) return 0;
    return (size_t)apm::back_shape(rows, cols).groups * apm::kSums * (size_t)cols * sizeof(float);
}

extern "C" int apm_norm_join_backward(const apm_norm_join* j, const apm_norm_join_grads* g, void* workspace, size_t workspace_bytes, void* stream) {
    return apm::guarded([&]() -> int { return apm::backward(j, g, workspace, workspace_bytes, stream); });
}
