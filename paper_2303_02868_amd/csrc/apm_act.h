// What the activation kernels share: eight elements at a time as they lie in memory, the 8-bit form, sums over the lanes
// that hold a row.  Device code, and the argument checks of the entry points.
#pragma once

#include "apm_internal.h"

namespace apm {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
// Any alignment: the target's unaligned access mode serves these with one access, so rows of odd widths and strides need no path of their own.
typedef u32x4 __attribute__((aligned(1))) u32x4_any;
typedef u32x2 __attribute__((aligned(1))) u32x2_any;

// (Functions of their own for each type: as an argument of a template it would lose its alignment.)
template <bool NT> __device__ __forceinline__ u32x4 load_at(const u32x4_any* p) { return NT ? __builtin_nontemporal_load(p) : *p; }
template <bool NT> __device__ __forceinline__ u32x2 load_at(const u32x2_any* p) { return NT ? __builtin_nontemporal_load(p) : *p; }
template <bool NT> __device__ __forceinline__ void store_at(u32x4 v, u32x4_any* p) {
    if constexpr (NT) __builtin_nontemporal_store(v, p);
    else *p = v;
}
template <bool NT> __device__ __forceinline__ void store_at(u32x2 v, u32x2_any* p) {
    if constexpr (NT) __builtin_nontemporal_store(v, p);
    else *p = v;
}

constexpr int kVec = 8;                          // elements a lane takes at a time: 16 bytes of bf16
constexpr int kQuad = APM_CKPT_BLOCK / kVec;     // neighbouring lanes that hold a block of the 8-bit form
static_assert(kQuad == 4, "a block is a quad of lanes");

struct bf16 {  // as a template argument; float is the other one
    uint16_t bits;
};

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __builtin_bit_cast(float, w & 0xffff0000u); }
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t to_bf16x2(float a, float b) {  // round to nearest, ties to even
    const bf16x2 v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ uint16_t to_bf16(float a) { return __builtin_bit_cast(uint16_t, (__bf16)a); }

// Eight elements as loaded.  n < 8 of them exist at the end of a row, the others read as zero.
template <class T> struct Raw;
template <> struct Raw<bf16> {
    u32x4 a;
    template <bool NT = false> __device__ __forceinline__ void load(const void* row, int col, int n) {
        const char* p = (const char*)row + (uint32_t)col * 2u;
        a = u32x4{0, 0, 0, 0};
        if (n >= kVec) {
            a = load_at<NT>((const u32x4_any*)p);
        } else {
#pragma unroll
            for (int i = 0; i < kVec; ++i)
                if (i < n) a[i / 2] |= (uint32_t)((const uint16_t*)p)[i] << (16 * (i & 1));
        }
    }
    __device__ __forceinline__ float operator[](int i) const { return (i & 1) ? bf16_hi(a[i / 2]) : bf16_lo(a[i / 2]); }
};
template <> struct Raw<float> {
    u32x4 a, b;
    template <bool NT = false> __device__ __forceinline__ void load(const void* row, int col, int n) {
        const char* p = (const char*)row + (int64_t)col * 4;  // past 32 bits from column 2^30 on
        a = b = u32x4{0, 0, 0, 0};
        if (n >= kVec) {
            a = load_at<NT>((const u32x4_any*)p);
            b = load_at<NT>((const u32x4_any*)p + 1);
        } else {
#pragma unroll
            for (int i = 0; i < kVec; ++i)
                if (i < n) {
                    if (i < 4) a[i & 3] = ((const uint32_t*)p)[i];
                    else b[i & 3] = ((const uint32_t*)p)[i];
                }
        }
    }
    __device__ __forceinline__ float operator[](int i) const { return __builtin_bit_cast(float, i < 4 ? a[i & 3] : b[i & 3]); }
};
template <class T, bool NT = false> __device__ __forceinline__ void store8(void* row, int col, int n, const float (&v)[kVec]) {
    char* p = (char*)row + (int64_t)col * (int64_t)sizeof(T);
    if constexpr (sizeof(T) == sizeof(float)) {
        if (n >= kVec) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                u32x4 w;
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = __builtin_bit_cast(uint32_t, v[4 * h + i]);
                store_at<NT>(w, (u32x4_any*)p + h);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kVec; ++i)
                if (i < n) ((float*)p)[i] = v[i];
        }
    } else {
        if (n >= kVec) {
            u32x4 w;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = to_bf16x2(v[2 * i], v[2 * i + 1]);
            store_at<NT>(w, (u32x4_any*)p);
        } else {
#pragma unroll
            for (int i = 0; i < kVec; ++i)
                if (i < n) ((uint16_t*)p)[i] = to_bf16(v[i]);
        }
    }
}
// One element whose type is known at run time (vectors of parameters and their gradients: a few per column, not per element).
__device__ __forceinline__ float load1(const void* p, int32_t dtype, int64_t i) {
    return dtype == APM_F32 ? ((const float*)p)[i] : bf16_lo(((const uint16_t*)p)[i]);
}
__device__ __forceinline__ void store1(void* p, int32_t dtype, int64_t i, float v) {
    if (dtype == APM_F32) ((float*)p)[i] = v;
    else ((uint16_t*)p)[i] = to_bf16(v);
}
// Eight of them: the loads are issued whatever the type is, and looked at when they are needed.
struct RawAny {
    u32x4 a, b;
    __device__ __forceinline__ void load(const void* row, int32_t dtype, int col, int n) {
        const bool wide = dtype == APM_F32;
        a = b = u32x4{0, 0, 0, 0};
        const char* p = (const char*)row + (uint32_t)col * (wide ? 4u : 2u);
        if (n >= kVec) {
            a = ((const u32x4_any*)p)[0];
            if (wide) b = ((const u32x4_any*)p)[1];
        } else if (wide) {
#pragma unroll
            for (int i = 0; i < kVec; ++i)
                if (i < n) {
                    if (i < 4) a[i & 3] = ((const uint32_t*)p)[i];
                    else b[i & 3] = ((const uint32_t*)p)[i];
                }
        } else {
#pragma unroll
            for (int i = 0; i < kVec; ++i)
                if (i < n) a[i / 2] |= (uint32_t)((const uint16_t*)p)[i] << (16 * (i & 1));
        }
    }
    __device__ __forceinline__ void get(int32_t dtype, float (&v)[kVec]) const {
        if (dtype == APM_F32) {
#pragma unroll
            for (int i = 0; i < kVec; ++i) v[i] = __builtin_bit_cast(float, i < 4 ? a[i & 3] : b[i & 3]);
        } else {
#pragma unroll
            for (int i = 0; i < kVec; ++i) v[i] = (i & 1) ? bf16_hi(a[i / 2]) : bf16_lo(a[i / 2]);
        }
    }
};

// A row as a buffer: what lies beyond it (or all of it, if there is no such row or matrix) reads as zero and is not written, so that every lane
// loads and stores without a branch, and nothing waits for more than it needs.  The bound is checked for each 32-bit word of an access by itself: an
// fp32 row may end anywhere.  Non-temporal: these streams are larger than the caches (gradients of a join of 8192 x 5120, fp32 stream, when this was chosen: 119 us
// with the default policy, 115 with non-temporal stores, 108.6 with loads too).
typedef __amdgpu_buffer_rsrc_t Rsrc;
constexpr int kNT = 2;
__device__ __forceinline__ Rsrc row_buffer(const void* data, int64_t byte_offset, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>((const char*)data + byte_offset), 0, data ? bytes : 0, 0x00027000);
}
template <int CACHE = kNT> __device__ __forceinline__ u32x4 load_b128(Rsrc r, uint32_t byte) {
    return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, (int)byte, 0, CACHE));
}
__device__ __forceinline__ u32x2 load_b64(Rsrc r, uint32_t byte) { return __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r, (int)byte, 0, kNT)); }

// A lane's eight columns.  fp32 takes two accesses of 16 bytes.  Each of them covers whole cache lines if the lower half of the wavefront's lanes takes
// first halves and the upper half second ones, of the lower half's columns and then of the upper half's; the halves then change places in
// registers (the same gradients: 119 us with each lane's own 32 bytes).
struct LaneCols {
    int col, n;      // n of the eight are there; 0 or less: none
    uint32_t whole;  // columns in whole vectors
    uint32_t at4;    // fp32: byte of the first access, the second is kStep4 behind it
    static constexpr uint32_t kStep4 = 1024;
    __device__ __forceinline__ void set(int first, int64_t cols) {
        const uint32_t lane = threadIdx.x % 64u;
        col = first;
        n = (int)min((int64_t)kVec, cols - first);
        whole = (uint32_t)cols / kVec * kVec;
        at4 = ((uint32_t)col - lane * kVec) * 4u + lane % 32u * 32u + lane / 32u * 16u;
    }
    __device__ __forceinline__ bool tail() const { return n > 0 && n < kVec; }
};
__device__ __forceinline__ void swap_halves(u32x4& a, u32x4& b) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const auto r = __builtin_amdgcn_permlane32_swap(a[i], b[i], false, false);
        a[i] = r[0], b[i] = r[1];
    }
}
// A row's last eight elements, n of which are wanted, moved down to the first places, zeros behind them
__device__ __forceinline__ void move_down(u32x4& w, int n) {
    const int by = kVec - n;
    uint64_t lo = (uint64_t)w[1] << 32 | w[0], hi = (uint64_t)w[3] << 32 | w[2];
    if (by & 4) lo = hi, hi = 0;
    const int s = (by & 3) * 16;
    lo = lo >> s | (hi << 1) << (63 - s);
    hi >>= s;
    w = u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
}
__device__ __forceinline__ void move_down(u32x2& w, int n) {
    const uint64_t v = ((uint64_t)w[1] << 32 | w[0]) >> (8 * (kVec - n));
    w = u32x2{(uint32_t)v, (uint32_t)(v >> 32)};
}

// The rest goes element by element, in loops and not unrolled: a call of few rows runs through a kernel's code once, and waits for that code.
__device__ __forceinline__ u32x4 load_short(const uint16_t* p, int n) {
    uint64_t lo = 0, hi = 0;
#pragma unroll 1
    for (int i = n - 1; i >= 0; --i) {
        hi = hi << 16 | lo >> 48;
        lo = lo << 16 | p[i];
    }
    return u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
}
__device__ __forceinline__ u32x2 load_short(const uint8_t* p, int n) {
    uint64_t w = 0;
#pragma unroll 1
    for (int i = n - 1; i >= 0; --i) w = w << 8 | p[i];
    return u32x2{(uint32_t)w, (uint32_t)(w >> 32)};
}
__device__ __forceinline__ void store_short(uint16_t* p, int n, u32x4 w) {
    uint64_t lo = (uint64_t)w[1] << 32 | w[0], hi = (uint64_t)w[3] << 32 | w[2];
#pragma unroll 1
    for (int i = 0; i < n; ++i) {
        p[i] = (uint16_t)lo;
        lo = lo >> 16 | hi << 48;
        hi >>= 16;
    }
}
__device__ __forceinline__ void store_short(uint8_t* p, int n, u32x2 w) {
    uint64_t v = (uint64_t)w[1] << 32 | w[0];
#pragma unroll 1
    for (int i = 0; i < n; ++i, v >>= 8) p[i] = (uint8_t)v;
}

// Row `row` of a matrix: load_row, and settle before the first look at it.  A bf16 row's last elements, fewer than eight, come as the end of the eight
// that end with the row, where it has eight, and not one by one: a branch and a trip to memory for each took gradients of 8000 x 1501 (RMS) 71 us and not 42.
template <int CACHE = kNT> __device__ __forceinline__ u32x4 load_bf16(const void* data, int64_t byte_offset, int64_t cols, bool there, const LaneCols& l) {
    const bool eight = cols >= kVec;
    const int from = l.tail() && eight ? (int)cols - kVec : l.col;
    u32x4 a = load_b128<CACHE>(row_buffer(data, byte_offset, there && eight ? (uint32_t)cols * 2u : 0u), (uint32_t)from * 2u);
    if (!eight && there && data && l.tail()) a = load_short((const uint16_t*)((const char*)data + byte_offset), l.n);
    return a;
}
__device__ __forceinline__ void settle_bf16(u32x4& a, const LaneCols& l, int64_t cols) {
    if (l.whole != (uint32_t)cols && cols >= kVec && l.tail()) move_down(a, l.n);
}
template <int CACHE = kNT> __device__ __forceinline__ void load_row(Raw<bf16>& x, const apm_matrix& m, int64_t row, int64_t cols, bool there, const LaneCols& l) {
    x.a = load_bf16<CACHE>(m.data, row * m.stride * 2, cols, there, l);
}
template <int CACHE = kNT> __device__ __forceinline__ void load_row(Raw<float>& x, const apm_matrix& m, int64_t row, int64_t cols, bool there, const LaneCols& l) {
    const Rsrc r = row_buffer(m.data, row * m.stride * 4, there ? (uint32_t)cols * 4u : 0u);
    x.a = load_b128<CACHE>(r, l.at4);
    x.b = load_b128<CACHE>(r, l.at4 + LaneCols::kStep4);
}
__device__ __forceinline__ void settle(Raw<bf16>& x, const LaneCols& l, int64_t cols) { settle_bf16(x.a, l, cols); }
__device__ __forceinline__ void settle(Raw<float>& x, const LaneCols&, int64_t) { swap_halves(x.a, x.b); }
// The same for eight columns of a vector of parameters, or of a gate, whose type is known at run time
struct RowAny {
    u32x4 a, b;
    __device__ __forceinline__ void load(const void* data, int64_t offset, int32_t dtype, int64_t cols, bool there, const LaneCols& l) {
        if (dtype == APM_F32) {
            const Rsrc r = row_buffer(data, offset * 4, there ? (uint32_t)cols * 4u : 0u);
            a = load_b128<0>(r, (uint32_t)l.col * 4u);
            b = load_b128<0>(r, (uint32_t)l.col * 4u + 16u);
        } else {
            a = load_bf16<0>(data, offset * 2, cols, there, l);
        }
    }
    __device__ __forceinline__ void get(int32_t dtype, int64_t cols, const LaneCols& l, float (&v)[kVec]) {
        if (dtype == APM_F32) {
#pragma unroll
            for (int i = 0; i < kVec; ++i) v[i] = __builtin_bit_cast(float, i < 4 ? a[i & 3] : b[i & 3]);
        } else {
            settle_bf16(a, l, cols);
#pragma unroll
            for (int i = 0; i < kVec; ++i) v[i] = (i & 1) ? bf16_hi(a[i / 2]) : bf16_lo(a[i / 2]);
        }
    }
};
template <class T, int CACHE = kNT> __device__ __forceinline__ void store_row(const apm_matrix& m, int64_t row, int64_t cols, bool there, const LaneCols& l, const float (&v)[kVec]) {
    if constexpr (sizeof(T) == sizeof(float)) {
        const Rsrc r = row_buffer(m.data, row * m.stride * 4, there ? (uint32_t)cols * 4u : 0u);
        u32x4 w[2];
#pragma unroll
        for (int i = 0; i < kVec; ++i) w[i / 4][i % 4] = __builtin_bit_cast(uint32_t, v[i]);
        swap_halves(w[0], w[1]);
        __builtin_amdgcn_raw_buffer_store_b128(w[0], r, (int)l.at4, 0, CACHE);
        __builtin_amdgcn_raw_buffer_store_b128(w[1], r, (int)(l.at4 + LaneCols::kStep4), 0, CACHE);
    } else {
        const Rsrc r = row_buffer(m.data, row * m.stride * 2, there ? l.whole * 2u : 0u);
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = to_bf16x2(v[2 * i], v[2 * i + 1]);
        __builtin_amdgcn_raw_buffer_store_b128(w, r, (int)((uint32_t)l.col * 2u), 0, CACHE);
        if (l.whole != (uint32_t)cols && there && m.data && l.tail()) store_short((uint16_t*)((char*)m.data + row * m.stride * 2) + l.col, l.n, w);
    }
}

// ---- the 8-bit form -----------------------------------------------------------------------------
// The lanes of a quad (four neighbours from a multiple of four on) hold a block, eight elements each, those beyond the row's end zero.
template <int CTRL> __device__ __forceinline__ uint32_t dpp_u32(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, CTRL, 0xf, 0xf, true);
}
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
    x = max(x, dpp_u32<0xB1>(x));  // lanes 1 0 3 2
    return max(x, dpp_u32<0x4E>(x));  // lanes 2 3 0 1
}
// The bits of |x| count up with it, infinities and NaN above all numbers, so the block's largest decides.  The exponent of the scale
// is that of the largest, one more where rounding would carry the largest out of range: from 127.5 / 64 on (I8), above 464 (F8).
__device__ __forceinline__ uint32_t scale_byte(uint32_t largest, int32_t format) {
    if (largest >= 0x7f800000u) return 255u;
    if (format == APM_CKPT_I8) return min((largest + 0x00010000u) >> 23, 254u);
    const uint32_t e = (largest + 0x0017ffffu) >> 23;
    return e > 8u ? e - 8u : 0u;
}
__device__ __forceinline__ u32x2 encode8(const float (&v)[kVec], int32_t format, uint32_t* scale) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < kVec; ++i) m = max(m, __builtin_bit_cast(uint32_t, v[i]) & 0x7fffffffu);
    const uint32_t s = scale_byte(quad_max(m), format);
    *scale = s;
    if (s == 255u) return u32x2{0u, 0u};
    u32x2 w;
    if (format == APM_CKPT_I8) {
        uint32_t q[kVec];
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            // Between 2^23 and 2^24 floats are the whole numbers, so this sum rounds to one; its low byte is that number's.
            const float x = __builtin_amdgcn_fmed3f(__builtin_amdgcn_ldexpf(v[i], 133 - (int)s), -127.0f, 127.0f);
            q[i] = __builtin_bit_cast(uint32_t, x + 12582912.0f);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t lo = __builtin_amdgcn_perm(q[4 * h + 1], q[4 * h], 0x0c0c0400u), hi = __builtin_amdgcn_perm(q[4 * h + 3], q[4 * h + 2], 0x04000c0cu);
            w[h] = lo | hi;
        }
    } else {
        float x[kVec];
#pragma unroll
        for (int i = 0; i < kVec; ++i) x[i] = __builtin_amdgcn_ldexpf(v[i], 127 - (int)s);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            int p = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * h], x[4 * h + 1], 0, false);
            w[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[4 * h + 2], x[4 * h + 3], p, true);
        }
    }
    return w;
}
// What an element of a block is multiplied by: a power of two, so that values are exact; NaN for the block that has none.
__device__ __forceinline__ float scale_of(uint32_t s, int32_t format) {
    const float m = __builtin_amdgcn_ldexpf(1.0f, (int)s - (format == APM_CKPT_I8 ? 133 : 127));
    return s == 255u ? __builtin_nanf("") : m;
}
typedef float f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void decode8(u32x2 w, float m, int32_t format, float (&v)[kVec]) {
    if (format == APM_CKPT_I8) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) v[i] = (float)(int8_t)(w[i / 4] >> (8 * (i & 3))) * m;
    } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[h], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[h], true);
            v[4 * h] = a[0] * m, v[4 * h + 1] = a[1] * m, v[4 * h + 2] = b[0] * m, v[4 * h + 3] = b[1] * m;
        }
    }
}
template <bool NT = false> __device__ __forceinline__ u32x2 load_q(const void* row, int col, int n) {
    const char* p = (const char*)row + (uint32_t)col;
    u32x2 w = {0u, 0u};
    if (n >= kVec) {
        w = load_at<NT>((const u32x2_any*)p);
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            if (i < n) w[i / 4] |= (uint32_t)((const uint8_t*)p)[i] << (8 * (i & 3));
    }
    return w;
}
template <bool NT = false> __device__ __forceinline__ void store_q(void* row, int col, int n, u32x2 w) {
    char* p = (char*)row + (uint32_t)col;
    if (n >= kVec) {
        store_at<NT>(w, (u32x2_any*)p);
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            if (i < n) ((uint8_t*)p)[i] = (uint8_t)(w[i / 4] >> (8 * (i & 3)));
    }
}

// A lane's eight bytes and its block's scale byte.
struct Kept {
    u32x2 q;
    uint32_t s;
    __device__ __forceinline__ void load(const apm_ckpt& c, int64_t row, int64_t cols, bool there, const LaneCols& l) {
        const uint32_t blocks = ((uint32_t)cols + APM_CKPT_BLOCK - 1) / APM_CKPT_BLOCK;
        const bool eight = cols >= kVec;
        const int from = l.tail() && eight ? (int)cols - kVec : l.col;
        q = load_b64(row_buffer(c.q, row * c.q_stride, there && eight ? (uint32_t)cols : 0u), (uint32_t)from);
        s = __builtin_amdgcn_raw_buffer_load_b8(row_buffer(c.q ? c.scale : nullptr, row * c.scale_stride, there ? blocks : 0u), l.col / APM_CKPT_BLOCK, 0, 0);
        if (!eight && there && c.q && l.tail()) q = load_short((const uint8_t*)c.q + row * c.q_stride, l.n);
    }
    __device__ __forceinline__ void settle(const LaneCols& l, int64_t cols) {
        if (l.whole != (uint32_t)cols && cols >= kVec && l.tail()) move_down(q, l.n);
    }
    __device__ __forceinline__ void get(int32_t format, float (&v)[kVec]) const { decode8(q, scale_of(s, format), format, v); }
};
// Encodes and stores a lane's eight columns; quads of lanes hold a block.
__device__ __forceinline__ void keep(const apm_ckpt& c, int64_t row, int64_t cols, bool there, const LaneCols& l, const float (&v)[kVec]) {
    uint32_t s;
    const u32x2 w = encode8(v, c.format, &s);
    __builtin_amdgcn_raw_buffer_store_b64(w, row_buffer(c.q, row * c.q_stride, there ? l.whole : 0u), l.col, 0, kNT);
    if (l.whole != (uint32_t)cols && there && l.tail()) store_short((uint8_t*)c.q + row * c.q_stride + l.col, l.n, w);
    if (threadIdx.x % kQuad == 0 && there && l.n > 0) ((uint8_t*)c.scale)[row * c.scale_stride + (uint32_t)l.col / APM_CKPT_BLOCK] = (uint8_t)s;
}

// ---- sums over a wavefront ----------------------------------------------------------------------
template <int CTRL> __device__ __forceinline__ float dpp_add(float x) {
    return x + __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float row_sum16(float x) {  // of 16 lanes, the same in each: rotated by 8, 4, 2, 1
    return dpp_add<0x121>(dpp_add<0x122>(dpp_add<0x124>(dpp_add<0x128>(x))));
}
// Rows 0 and 1, 2 and 3 of 16 lanes, or the halves, change places between two copies, whose sum then has both.  The copy is made in a
// statement of its own: given one value twice, the compiler takes the first result for both.
template <bool HALVES> __device__ __forceinline__ float swap_add(float x) {
    uint32_t a = __builtin_bit_cast(uint32_t, x), b;
    asm("v_mov_b32 %0, %1" : "=v"(b) : "v"(a));
    const auto r = HALVES ? __builtin_amdgcn_permlane32_swap(a, b, false, false) : __builtin_amdgcn_permlane16_swap(a, b, false, false);
    return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
}
__device__ __forceinline__ float wave_sum(float x) { return swap_add<true>(swap_add<false>(row_sum16(x))); }  // the same in every lane

// What lanes of a wavefront hand each other through LDS: its accesses are carried out in order, so it is the compiler's order that counts.
__device__ __forceinline__ void among_lanes() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// ---- argument checks ----------------------------------------------------------------------------
int check_matrix(const char* name, const apm_matrix& m, int64_t rows, int64_t cols, bool written);
int check_vector(const char* name, const apm_vector& v);
int check_ckpt(const char* name, const apm_ckpt& c, int64_t rows, int64_t cols, bool written);

inline int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace apm
