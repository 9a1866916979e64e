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
    __device__ __forceinline__ void load(const void* row, int col, int n) {
        const char* p = (const char*)row + (int64_t)col * 2;
        a = u32x4{0, 0, 0, 0};
        if (n >= kVec) {
            a = *(const u32x4_any*)p;
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
    __device__ __forceinline__ void load(const void* row, int col, int n) {
        const char* p = (const char*)row + (int64_t)col * 4;
        a = b = u32x4{0, 0, 0, 0};
        if (n >= kVec) {
            a = ((const u32x4_any*)p)[0];
            b = ((const u32x4_any*)p)[1];
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
template <class T> __device__ __forceinline__ void store8(void* row, int col, int n, const float (&v)[kVec]) {
    char* p = (char*)row + (int64_t)col * (int64_t)sizeof(T);
    if constexpr (sizeof(T) == sizeof(float)) {
        if (n >= kVec) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                u32x4 w;
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = __builtin_bit_cast(uint32_t, v[4 * h + i]);
                ((u32x4_any*)p)[h] = w;
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
            *(u32x4_any*)p = w;
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
        const char* p = (const char*)row + (int64_t)col * (wide ? 4 : 2);
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
__device__ __forceinline__ u32x2 load_q(const void* row, int col, int n) {
    const char* p = (const char*)row + col;
    u32x2 w = {0u, 0u};
    if (n >= kVec) {
        w = *(const u32x2_any*)p;
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            if (i < n) w[i / 4] |= (uint32_t)((const uint8_t*)p)[i] << (8 * (i & 3));
    }
    return w;
}
__device__ __forceinline__ void store_q(void* row, int col, int n, u32x2 w) {
    char* p = (char*)row + col;
    if (n >= kVec) {
        *(u32x2_any*)p = w;
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            if (i < n) ((uint8_t*)p)[i] = (uint8_t)(w[i / 4] >> (8 * (i & 3)));
    }
}

// ---- sums over a wavefront ----------------------------------------------------------------------
template <int CTRL, int ROWS> __device__ __forceinline__ float dpp_add(float x) {
    return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float wave_sum(float x) {  // the same in every lane
    x = dpp_add<0x111, 0xf>(x);  // lane - 1, - 2, - 4, - 8 of 16: lane 15 has the row's
    x = dpp_add<0x112, 0xf>(x);
    x = dpp_add<0x114, 0xf>(x);
    x = dpp_add<0x118, 0xf>(x);
    x = dpp_add<0x142, 0xa>(x);  // rows 0 into 1, 2 into 3
    x = dpp_add<0x143, 0xc>(x);  // row 1 into 2 and 3
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}

// ---- argument checks ----------------------------------------------------------------------------
int check_matrix(const char* name, const apm_matrix& m, int64_t rows, int64_t cols, bool written);
int check_vector(const char* name, const apm_vector& v);
int check_ckpt(const char* name, const apm_ckpt& c, int64_t rows, int64_t cols, bool written);

inline int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace apm
