// Where one block of a residual network ends and the next begins: y = scale x + gate post(branch), n = pre(y), with both
// normalised tensors kept in 8 bits, and the gradients out of those.  HBM-bound in both directions (bf16: 10 B/element
// and the scales, forward x, branch, y, n and two bytes, backward dy, dn, two bytes, dx, dbranch), so a row is read once
// and stays in registers between its sums: 16 elements a lane, by one wavefront up to 1024 columns, else by as many as it takes.
#include <algorithm>

#include "apm_act.h"

namespace apm {
namespace {

constexpr int kWave = 64, kMaxWaves = 16, kMaxThreads = kWave * kMaxWaves;
constexpr int kVecs = 2;                          // vectors of a lane
constexpr int kWaveCols = kWave * kVec * kVecs;   // that one wavefront holds
static_assert(kWaveCols * kMaxWaves == APM_JOIN_MAX_COLS, "a row fits the largest workgroup");

struct JoinArgs {
    apm_norm_join j;
    float scale, eps_pre, eps_post, inv_cols;
};

// Sums over the lanes that hold a row: a wavefront, or `waves` consecutive ones of the workgroup from `first` on, whose sums go through
// `slots` (of the whole workgroup's wavefronts, for this sum alone until the next barrier but one).
template <bool WAVE, int N>
__device__ __forceinline__ void row_sums(float (&x)[N], float* slots, int first, int waves) {
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = wave_sum(x[k]);
    if constexpr (!WAVE) {
        if (threadIdx.x % kWave == 0)
#pragma unroll
            for (int k = 0; k < N; ++k) slots[k * kMaxWaves + threadIdx.x / kWave] = x[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) {
            float s = 0.0f;
            for (int w = first; w < first + waves; ++w) s += slots[k * kMaxWaves + w];
            x[k] = s;
        }
    }
}

// z becomes hat(z); elements beyond the row's end are zero before and after.
template <bool WAVE>
__device__ __forceinline__ float normalise(float (&z)[kVecs][kVec], const int (&n)[kVecs], int32_t kind, float eps, float inv_cols, float* slots, int waves) {
    if (kind == APM_NORM_NONE) return 1.0f;
    if (kind == APM_NORM_LAYER) {
        float s[1] = {0.0f};
#pragma unroll
        for (int v = 0; v < kVecs; ++v)
#pragma unroll
            for (int i = 0; i < kVec; ++i) s[0] += z[v][i];
        row_sums<WAVE>(s, slots, 0, waves);
        const float mean = s[0] * inv_cols;
#pragma unroll
        for (int v = 0; v < kVecs; ++v)
#pragma unroll
            for (int i = 0; i < kVec; ++i) z[v][i] = i < n[v] ? z[v][i] - mean : 0.0f;
    }
    float q[1] = {0.0f};
#pragma unroll
    for (int v = 0; v < kVecs; ++v)
#pragma unroll
        for (int i = 0; i < kVec; ++i) q[0] = fmaf(z[v][i], z[v][i], q[0]);
    row_sums<WAVE>(q, slots + kMaxWaves, 0, waves);
    const float r = 1.0f / sqrtf(fmaf(q[0], inv_cols, eps));
#pragma unroll
    for (int v = 0; v < kVecs; ++v)
#pragma unroll
        for (int i = 0; i < kVec; ++i) z[v][i] *= r;
    return r;
}

__device__ __forceinline__ void keep(const apm_ckpt& c, int64_t row, int col, int n, const float (&z)[kVec]) {
    uint32_t s;
    const u32x2 w = encode8(z, c.format, &s);
    store_q((char*)c.q + row * c.q_stride, col, n, w);
    if (threadIdx.x % kQuad == 0 && n > 0) ((uint8_t*)c.scale)[row * c.scale_stride + col / APM_CKPT_BLOCK] = (uint8_t)s;
}

// weight and bias, where they are given
__device__ __forceinline__ void affine(const apm_norm& norm, int col, int n, const float (&z)[kVec], float (&out)[kVec]) {
    RawAny w, b;
    if (norm.weight.data) w.load(norm.weight.data, norm.weight.dtype, col, n);
    if (norm.bias.data) b.load(norm.bias.data, norm.bias.dtype, col, n);
#pragma unroll
    for (int i = 0; i < kVec; ++i) out[i] = z[i];
    float p[kVec];
    if (norm.weight.data) {
        w.get(norm.weight.dtype, p);
#pragma unroll
        for (int i = 0; i < kVec; ++i) out[i] *= p[i];
    }
    if (norm.bias.data) {
        b.get(norm.bias.dtype, p);
#pragma unroll
        for (int i = 0; i < kVec; ++i) out[i] += p[i];
    }
}

__device__ __forceinline__ const char* row_of(const apm_matrix& m, int64_t row) {
    return (const char*)m.data + row * m.stride * (m.dtype == APM_F32 ? 4 : 2);
}

constexpr int kRowsPerGroup = 4;  // of one wavefront each

template <class R, class A, bool WAVE>
__global__ __launch_bounds__(WAVE ? kWave * kRowsPerGroup : kMaxThreads) void apm_join_forward_kernel(JoinArgs a) {
    __shared__ float slots[WAVE ? 1 : 4 * kMaxWaves];
    const apm_norm_join& j = a.j;
    const int lane = WAVE ? (int)threadIdx.x % kWave : (int)threadIdx.x, lanes = WAVE ? kWave : (int)blockDim.x, waves = lanes / kWave;
    int64_t row = blockIdx.x;
    if constexpr (WAVE) {
        row = row * kRowsPerGroup + __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
        if (row >= j.rows) return;
    }
    int col[kVecs], n[kVecs];
    Raw<R> x[kVecs];
    Raw<A> b[kVecs];
#pragma unroll
    for (int v = 0; v < kVecs; ++v) {
        col[v] = (v * lanes + lane) * kVec;
        n[v] = (int)min((int64_t)kVec, j.cols - col[v]);
        x[v].load((const char*)j.x.data + row * j.x.stride * (int64_t)sizeof(R), col[v], n[v]);
        if (j.branch.data) b[v].load((const char*)j.branch.data + row * j.branch.stride * (int64_t)sizeof(A), col[v], n[v]);
    }
    float y[kVecs][kVec];
#pragma unroll
    for (int v = 0; v < kVecs; ++v)
#pragma unroll
        for (int i = 0; i < kVec; ++i) y[v][i] = a.scale * x[v][i];
    if (j.branch.data) {
        float z[kVecs][kVec];
#pragma unroll
        for (int v = 0; v < kVecs; ++v)
#pragma unroll
            for (int i = 0; i < kVec; ++i) z[v][i] = b[v][i];
        const float r = normalise<WAVE>(z, n, j.post.kind, a.eps_post, a.inv_cols, slots, waves);
        if (j.post.rstd && lane == 0) j.post.rstd[row] = r;
        const float token = j.gate_kind == APM_GATE_TOKEN ? load1(j.gate.data, j.gate.dtype, row * j.gate.stride) : 1.0f;
#pragma unroll
        for (int v = 0; v < kVecs; ++v) {
            if (j.post.ckpt.q) keep(j.post.ckpt, row, col[v], n[v], z[v]);
            float c[kVec];
            affine(j.post, col[v], n[v], z[v], c);
            if (j.gate_kind == APM_GATE_CHANNEL || j.gate_kind == APM_GATE_FULL) {
                RawAny raw;
                raw.load(j.gate_kind == APM_GATE_FULL ? row_of(j.gate, row) : (const char*)j.gate.data, j.gate.dtype, col[v], n[v]);
                float g[kVec];
                raw.get(j.gate.dtype, g);
#pragma unroll
                for (int i = 0; i < kVec; ++i) y[v][i] = fmaf(g[i], c[i], y[v][i]);
            } else {
#pragma unroll
                for (int i = 0; i < kVec; ++i) y[v][i] = fmaf(token, c[i], y[v][i]);
            }
        }
    }
    if (j.y.data) {
#pragma unroll
        for (int v = 0; v < kVecs; ++v) store8<R>((char*)j.y.data + row * j.y.stride * (int64_t)sizeof(R), col[v], n[v], y[v]);
    }
    if (!j.n.data && !j.pre.ckpt.q && !j.pre.rstd) return;
    const float r = normalise<WAVE>(y, n, j.pre.kind, a.eps_pre, a.inv_cols, slots + 2 * kMaxWaves * (WAVE ? 0 : 1), waves);
    if (j.pre.rstd && lane == 0) j.pre.rstd[row] = r;
#pragma unroll
    for (int v = 0; v < kVecs; ++v) {
        if (j.pre.ckpt.q) keep(j.pre.ckpt, row, col[v], n[v], y[v]);
        if (j.n.data) {
            float o[kVec];
            affine(j.pre, col[v], n[v], y[v], o);
            store8<A>((char*)j.n.data + row * j.n.stride * (int64_t)sizeof(A), col[v], n[v], o);
        }
    }
}

// ---- backward -----------------------------------------------------------------------------------
// Sums over rows: every team of lanes (a wavefront, or the wavefronts that hold a row) adds its rows up in registers, a workgroup's teams are
// added in LDS, the workgroups' sums in the workspace are added by a second kernel, all in one order.
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
    u32x2 q1[VECS], q2[VECS];
    uint32_t s1[VECS], s2[VECS];
    float r1, r2, token;
    __device__ __forceinline__ void load(const BackArgs& a, int64_t row, const int (&col)[VECS], const int (&count)[VECS]) {
        const bool there = row < a.j.rows;
        r1 = there && a.j.pre.kind != APM_NORM_NONE ? a.j.pre.rstd[row] : 1.0f;
        r2 = there && a.j.post.kind != APM_NORM_NONE && a.j.post.rstd ? a.j.post.rstd[row] : 1.0f;
        token = there && a.j.gate_kind == APM_GATE_TOKEN ? load1(a.j.gate.data, a.j.gate.dtype, row * a.j.gate.stride) : 1.0f;
#pragma unroll
        for (int v = 0; v < VECS; ++v) {
            const int n = there ? count[v] : 0;
            dy[v].load((const char*)a.g.dy.data + row * a.g.dy.stride * (int64_t)sizeof(R), col[v], a.g.dy.data ? n : 0);
            dn[v].load((const char*)a.g.dn.data + row * a.g.dn.stride * (int64_t)sizeof(A), col[v], a.g.dn.data ? n : 0);
            const bool k1 = a.j.pre.ckpt.q && n > 0, k2 = a.j.post.ckpt.q && n > 0;
            q1[v] = load_q((const char*)a.j.pre.ckpt.q + row * a.j.pre.ckpt.q_stride, col[v], k1 ? n : 0);
            q2[v] = load_q((const char*)a.j.post.ckpt.q + row * a.j.post.ckpt.q_stride, col[v], k2 ? n : 0);
            s1[v] = k1 ? ((const uint8_t*)a.j.pre.ckpt.scale)[row * a.j.pre.ckpt.scale_stride + col[v] / APM_CKPT_BLOCK] : 0u;
            s2[v] = k2 ? ((const uint8_t*)a.j.post.ckpt.scale)[row * a.j.post.ckpt.scale_stride + col[v] / APM_CKPT_BLOCK] : 0u;
        }
    }
};

__device__ __forceinline__ void load_vector(const apm_vector& p, int col, int n, float (&v)[kVec], float none) {
    if (p.data) {
        RawAny raw;
        raw.load(p.data, p.dtype, col, n);
        raw.get(p.dtype, v);
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = none;
    }
}

template <class R, class A, int VECS, bool WAVE, bool BIAS>
__global__ __launch_bounds__(kMaxThreads) void apm_join_backward_kernel(BackArgs a) {
    extern __shared__ float lds[];  // 2 x 5 sums of every wavefront while rows are walked, then the teams' sums
    const apm_norm_join& j = a.j;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const int waves = WAVE ? 1 : a.waves, team = wave / waves, first = team * waves;
    const int lanes = waves * kWave, lane = (int)threadIdx.x - first * kWave;
    int col[VECS], n[VECS];
#pragma unroll
    for (int v = 0; v < VECS; ++v) {
        col[v] = (v * lanes + lane) * kVec;
        n[v] = (int)min((int64_t)kVec, j.cols - col[v]);
    }
    float acc[BIAS ? 4 : 2][VECS][kVec];
#pragma unroll
    for (int k = 0; k < (BIAS ? 4 : 2); ++k)
#pragma unroll
        for (int v = 0; v < VECS; ++v)
#pragma unroll
            for (int i = 0; i < kVec; ++i) acc[k][v][i] = 0.0f;
    const bool pre = a.g.dn.data != nullptr;
    const int64_t step = (int64_t)gridDim.x * a.teams;
    int64_t row = (int64_t)blockIdx.x * a.teams + team;
    const int64_t begin = (int64_t)blockIdx.x * a.teams;  // the workgroup's first row: all its wavefronts walk as often
    RowRaw<R, A, VECS> next;
    next.load(a, row, col, n);
    int turn = 0;
    for (int64_t at = begin; at < j.rows; at += step, row += step, turn ^= 1) {
        const RowRaw<R, A, VECS> cur = next;
        const bool there = row < j.rows;
        if (at + step < j.rows) next.load(a, row + step, col, n);
        float* slots = lds + turn * 5 * kMaxWaves;
        float D[VECS][kVec];
        {
            float z[VECS][kVec], t[VECS][kVec], s[2] = {0.0f, 0.0f};
#pragma unroll
            for (int v = 0; v < VECS; ++v) {
                decode8(cur.q1[v], scale_of(cur.s1[v], j.pre.ckpt.format), j.pre.ckpt.format, z[v]);
                float w[kVec];
                load_vector(j.pre.weight, col[v], n[v], w, 1.0f);
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    const float dn = cur.dn[v][i];
                    t[v][i] = dn * w[i];
                    s[0] = fmaf(t[v][i], z[v][i], s[0]);
                    s[1] += t[v][i];
                    acc[0][v][i] = fmaf(dn, z[v][i], acc[0][v][i]);
                    if constexpr (BIAS) acc[2][v][i] += dn;
                }
            }
            if (pre && j.pre.kind != APM_NORM_NONE) {
                row_sums<WAVE>(s, slots, first, waves);
                const float k = s[0] * a.inv_cols, m = j.pre.kind == APM_NORM_LAYER ? s[1] * a.inv_cols : 0.0f;
#pragma unroll
                for (int v = 0; v < VECS; ++v)
#pragma unroll
                    for (int i = 0; i < kVec; ++i) t[v][i] = cur.r1 * (t[v][i] - fmaf(z[v][i], k, m));
            }
#pragma unroll
            for (int v = 0; v < VECS; ++v) {
                const int count = there ? n[v] : 0;
                float o[kVec];
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    D[v][i] = i < count ? cur.dy[v][i] + t[v][i] : 0.0f;
                    o[i] = a.scale * D[v][i];
                }
                if (a.g.dx.data) store8<R>((char*)a.g.dx.data + row * a.g.dx.stride * (int64_t)sizeof(R), col[v], count, o);
            }
        }
        {
            float z[VECS][kVec], s[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int v = 0; v < VECS; ++v) {
                const int count = there ? n[v] : 0;
                decode8(cur.q2[v], scale_of(cur.s2[v], j.post.ckpt.format), j.post.ckpt.format, z[v]);
                float w[kVec], g[kVec];
                load_vector(j.post.weight, col[v], n[v], w, 1.0f);
                if (j.gate_kind == APM_GATE_TOKEN || (j.gate_kind == APM_GATE_FULL && a.g.dgate.data)) {
                    float b[kVec], o[kVec];
                    load_vector(j.post.bias, col[v], n[v], b, 0.0f);
#pragma unroll
                    for (int i = 0; i < kVec; ++i) {
                        o[i] = D[v][i] * fmaf(z[v][i], w[i], b[i]);
                        s[2] += i < count ? o[i] : 0.0f;
                    }
                    if (j.gate_kind == APM_GATE_FULL) {
                        char* p = (char*)a.g.dgate.data + row * a.g.dgate.stride * (a.g.dgate.dtype == APM_F32 ? 4 : 2);
                        if (a.g.dgate.dtype == APM_F32) store8<float>(p, col[v], count, o);
                        else store8<bf16>(p, col[v], count, o);
                    }
                }
#pragma unroll
                for (int i = 0; i < kVec; ++i) g[i] = cur.token;
                if (j.gate_kind == APM_GATE_CHANNEL || j.gate_kind == APM_GATE_FULL) {
                    RawAny raw;
                    raw.load(j.gate_kind == APM_GATE_FULL ? row_of(j.gate, row) : (const char*)j.gate.data, j.gate.dtype, col[v], count);
                    raw.get(j.gate.dtype, g);
                }
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    const float dc = D[v][i] * g[i], summed = j.gate_kind == APM_GATE_CHANNEL ? D[v][i] : dc;
                    acc[1][v][i] = fmaf(summed, z[v][i], acc[1][v][i]);
                    if constexpr (BIAS) acc[3][v][i] += summed;
                    D[v][i] = dc * w[i];
                    s[0] = fmaf(D[v][i], z[v][i], s[0]);
                    s[1] += D[v][i];
                }
            }
            const bool through = a.g.dbranch.data && j.post.kind != APM_NORM_NONE;
            if (through || j.gate_kind == APM_GATE_TOKEN) {
                row_sums<WAVE>(s, slots + 2 * kMaxWaves, first, waves);
                if (j.gate_kind == APM_GATE_TOKEN && a.g.dgate.data && lane == 0 && there) store1(a.g.dgate.data, a.g.dgate.dtype, row * a.g.dgate.stride, s[2]);
            }
            if (a.g.dbranch.data) {
                const float k = s[0] * a.inv_cols, m = j.post.kind == APM_NORM_LAYER ? s[1] * a.inv_cols : 0.0f;
#pragma unroll
                for (int v = 0; v < VECS; ++v) {
                    float o[kVec];
#pragma unroll
                    for (int i = 0; i < kVec; ++i) o[i] = through ? cur.r2 * (D[v][i] - fmaf(z[v][i], k, m)) : D[v][i];
                    store8<A>((char*)a.g.dbranch.data + row * a.g.dbranch.stride * (int64_t)sizeof(A), col[v], there ? n[v] : 0, o);
                }
            }
        }
    }
    // The teams' sums.  The lane's 16 columns lie in LDS as in a row.
    const int64_t cap = (int64_t)lanes * kVec * VECS;
    float* mine = a.part + (int64_t)blockIdx.x * kSums * j.cols;
#pragma unroll
    for (int k = 0; k < (BIAS ? 4 : 2); ++k) {
        __syncthreads();
#pragma unroll
        for (int v = 0; v < VECS; ++v)
#pragma unroll
            for (int i = 0; i < kVec; ++i) lds[team * cap + col[v] + i] = acc[k][v][i];
        __syncthreads();
        const int sum = k == 0 ? kDnHat : k == 1 ? kDHat : k == 2 ? kDn : kD;
        for (int64_t c = threadIdx.x; c < j.cols; c += blockDim.x) {
            float s = 0.0f;
            for (int m = 0; m < a.teams; ++m) s += lds[m * cap + c];
            mine[sum * j.cols + c] = s;
        }
    }
    if (gridDim.x == 1) {
        for (int64_t c = threadIdx.x; c < j.cols; c += blockDim.x) {  // what this thread itself wrote
            float s[kSums] = {mine[kDnHat * j.cols + c], 0.0f, mine[kDHat * j.cols + c], 0.0f};
            if constexpr (BIAS) s[kDn] = mine[kDn * j.cols + c], s[kD] = mine[kD * j.cols + c];
            finish_column(j, a.g, c, s);
        }
    }
}

// The workgroups' sums of 32 columns: 32 lanes side by side, as many parts at a time.
constexpr int kSide = 32;
template <bool BIAS>
__global__ __launch_bounds__(kSide * kSide) void apm_join_sums_kernel(apm_norm_join j, apm_norm_join_grads g, const float* part, int32_t parts) {
    __shared__ float lds[kSide][kSide + 1];
    const int x = (int)threadIdx.x % kSide, y = (int)threadIdx.x / kSide;
    const int64_t c = (int64_t)blockIdx.x * kSide + x;
    float s[kSums] = {};
#pragma unroll
    for (int k = 0; k < kSums; ++k) {
        if (!BIAS && (k == kDn || k == kD)) continue;
        float t = 0.0f;
        if (c < j.cols)
            for (int32_t p = y; p < parts; p += kSide) t += part[((int64_t)p * kSums + k) * j.cols + c];
        __syncthreads();
        lds[y][x] = t;
        __syncthreads();
        if (y == 0)
            for (int i = 0; i < kSide; ++i) s[k] += lds[i][x];
    }
    if (y == 0 && c < j.cols) finish_column(j, g, c, s);
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
    if (rc == APM_OK && j.gate.data) rc = check_matrix("gate", j.gate, j.rows, j.cols, false);
    return rc;
}

// Types of the residual stream and of what goes in and out of blocks.
int check_types(const apm_matrix& res, const apm_matrix& act) {
    if (res.data && act.data && res.dtype == APM_BF16 && act.dtype == APM_F32)
        return fail(APM_EINVAL, "a bf16 residual stream with fp32 activations is not supported");
    return APM_OK;
}

int waves_of(int64_t cols) { return (int)div_up(cols, kWaveCols); }

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
    if (j.rows > (int64_t)1 << 31) return fail(APM_EINVAL, "too many rows");
    JoinArgs a{j, (float)j.residual_scale, (float)j.pre.eps, (float)j.post.eps, (float)(1.0 / (double)j.cols)};
    const int waves = waves_of(j.cols);
    with_types(j.x.dtype, act.data ? act.dtype : APM_BF16, [&](auto r, auto t) {
        using R = decltype(r);
        using A = decltype(t);
        const hipStream_t s = (hipStream_t)stream;
        if (waves == 1)
            hipLaunchKernelGGL((apm_join_forward_kernel<R, A, true>), dim3((unsigned)div_up(j.rows, kRowsPerGroup)), dim3(kWave * kRowsPerGroup), 0, s, a);
        else
            hipLaunchKernelGGL((apm_join_forward_kernel<R, A, false>), dim3((unsigned)j.rows), dim3((unsigned)(waves * kWave)), 0, s, a);
    });
    APM_HIP(hipGetLastError());
    return APM_OK;
}

// How many workgroups walk the rows, and with how many teams: one workgroup a CU.
constexpr int64_t kGroups = 256;
struct BackShape {
    int vecs, waves, teams;
    int64_t groups;
};
BackShape back_shape(int64_t rows, int64_t cols) {
    BackShape b;
    b.vecs = cols <= (int64_t)kMaxThreads * kVec ? 1 : 2;
    b.waves = (int)div_up(cols, kWave * kVec * b.vecs);
    b.teams = kMaxWaves / b.waves;
    b.groups = std::max<int64_t>(1, std::min(kGroups, div_up(rows, b.teams)));
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
    if (!g.dn.data) a.j.pre.kind = APM_NORM_NONE;
    if (j.rows > 0 && g.dbranch.data && j.post.kind != APM_NORM_NONE && !j.post.rstd) return fail(APM_EINVAL, "post.rstd is missing");
    if (workspace_bytes < apm_norm_join_workspace_bytes(j.rows, j.cols)) return fail(APM_ENOMEM, "the workspace is too small");
    if (!workspace || (uintptr_t)workspace % 16 != 0) return fail(APM_EINVAL, "the workspace is missing or not aligned to 16 bytes");
    const BackShape b = back_shape(j.rows, j.cols);
    a.waves = b.waves, a.teams = b.teams;
    const bool bias = g.dpre_bias.data || g.dpost_bias.data || (g.dgate.data && j.gate_kind == APM_GATE_CHANNEL && j.post.bias.data);
    const bool sums = bias || g.dpre_weight.data || g.dpost_weight.data || (g.dgate.data && j.gate_kind == APM_GATE_CHANNEL);
    const hipStream_t s = (hipStream_t)stream;
    const dim3 grid((unsigned)b.groups), block((unsigned)(b.teams * b.waves * kWave));
    const size_t shared = std::max<size_t>((size_t)block.x * kVec * b.vecs, 2 * 5 * kMaxWaves) * sizeof(float);
    with_types(res.data ? res.dtype : act.data ? act.dtype : APM_BF16, act.data ? act.dtype : APM_BF16, [&](auto r, auto t) {
        using R = decltype(r);
        using A = decltype(t);
        auto start = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, shared, s, a); };
        if (b.waves == 1) bias ? start(apm_join_backward_kernel<R, A, 1, true, true>) : start(apm_join_backward_kernel<R, A, 1, true, false>);
        else if (b.vecs == 1) bias ? start(apm_join_backward_kernel<R, A, 1, false, true>) : start(apm_join_backward_kernel<R, A, 1, false, false>);
        else bias ? start(apm_join_backward_kernel<R, A, 2, false, true>) : start(apm_join_backward_kernel<R, A, 2, false, false>);
    });
    APM_HIP(hipGetLastError());
    if (b.groups > 1 && sums) {
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
