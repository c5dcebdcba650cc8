// What the learner's operators share on the device: rows of fp32, binary16 or bfloat16 values that start at any element, and the
// two block formats (32 values along a row share one power of two).
#pragma once
#include <type_traits>

#include "common.hpp"

namespace aq {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef float v4f32 __attribute__((ext_vector_type(4)));
typedef float v2f32 __attribute__((ext_vector_type(2)));
typedef bf16_t v2bf16 __attribute__((ext_vector_type(2)));
typedef bf16_t v8bf16 __attribute__((ext_vector_type(8)));
typedef f16_t v2f16 __attribute__((ext_vector_type(2)));
// rows start at any element of their type (the hardware takes vector loads and stores at any address)
typedef v4u v4u_any __attribute__((aligned(2)));
typedef v2u v2u_any __attribute__((aligned(2)));

// ---- eight consecutive values as they lie in memory
template <class T>
struct Piece {
    static constexpr int kWords = 2 * (int)sizeof(T);
    uint32_t w[kWords];

    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = 0;
    }
    // all eight
    __device__ __forceinline__ void load_all(const T* __restrict__ p) {
#pragma unroll
        for (int i = 0; i < kWords; i += 4) {
            const v4u q = *(const v4u_any*)((const uint32_t AQ_GLOBAL*)p + i);
#pragma unroll
            for (int j = 0; j < 4; ++j) w[i + j] = q[j];
        }
    }
    // the first n (any number; zeros behind them)
    __device__ __forceinline__ void load(const T* __restrict__ p, int n) {
        if (n >= 8) {
            load_all(p);
            return;
        }
        zero();
        if (n > 0) load_some(p, n);
    }
    // The same of a row that has `before` values in front of these, to be settled before use: 16-bit values that a row ends among
    // come as its last eight, in one load that nothing waits for (value by value LayerNorm's gradients of 65536 x 501 took 71 us
    // for 59).
    __device__ __forceinline__ void request(const T* __restrict__ p, int n, int before) {
        if (n >= 8) {
            load_all(p);
        } else if (sizeof(T) == 2 && n > 0 && before + n >= 8) {
            load_all(p - (8 - n));
        } else {
            zero();
            if (n > 0) load_some(p, n);
        }
    }
    __device__ __forceinline__ void settle(int n, int before) {
        if constexpr (sizeof(T) == 2) {
            if (n > 0 && n < 8 && before + n >= 8) {
                const int skip = 8 - n;
                if (skip & 4) {
                    w[0] = w[2], w[1] = w[3], w[2] = 0, w[3] = 0;
                }
                if (skip & 2) {
                    w[0] = w[1], w[1] = w[2], w[2] = w[3], w[3] = 0;
                }
                if (skip & 1) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[i] = __builtin_amdgcn_alignbit(i < 3 ? w[i < 3 ? i + 1 : 0] : 0, w[i], 16);
                }
            }
        }
    }
    __device__ __forceinline__ void load_some(const T* __restrict__ p, int n) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) {
                if constexpr (sizeof(T) == 4) w[j] = ((const uint32_t*)p)[j];
                else w[j / 2] |= (uint32_t)((const uint16_t*)p)[j] << (16 * (j & 1));
            }
    }
    __device__ __forceinline__ void store(T* __restrict__ p, int n) const {
        if (n >= 8) {
#pragma unroll
            for (int i = 0; i < kWords; i += 4) *(v4u_any*)((uint32_t AQ_GLOBAL*)p + i) = (v4u){w[i], w[i + 1], w[i + 2], w[i + 3]};
            return;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) {
                if constexpr (sizeof(T) == 4) ((uint32_t*)p)[j] = w[j];
                else ((uint16_t*)p)[j] = (uint16_t)(w[j / 2] >> (16 * (j & 1)));
            }
    }
    __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if constexpr (std::is_same<T, float>::value) v[j] = __uint_as_float(w[j]);
            else if constexpr (std::is_same<T, bf16_t>::value) v[j] = __uint_as_float(j & 1 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
            else v[j] = (float)__builtin_bit_cast(v2f16, w[j / 2])[j & 1];
        }
    }
    // each rounded once, to nearest even
    __device__ __forceinline__ void set(const float (&v)[8]) {
        if constexpr (std::is_same<T, float>::value) {
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = __float_as_uint(v[j]);
        } else {
            typedef T v2 __attribute__((ext_vector_type(2)));
#pragma unroll
            for (int j = 0; j < 8; j += 2) w[j / 2] = __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f32{v[j], v[j + 1]}), v2));
        }
    }
};

// ---- blocks of 32 values: lanes 4 i .. 4 i + 3 hold one, eight values each
// The largest magnitude's bits as fp32's, found among whole numbers so that NaNs and infinities win; 16-bit values two at a time.
typedef uint16_t v2u16 __attribute__((ext_vector_type(2)));
template <class T>
__device__ __forceinline__ uint32_t most_of(const Piece<T>& p) {
    if constexpr (sizeof(T) == 4) {
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t b = p.w[j] & 0x7fffffffu;
            m = b > m ? b : m;
        }
        return m;
    } else {
        v2u16 m{0, 0};
#pragma unroll
        for (int j = 0; j < 4; ++j) m = __builtin_elementwise_max(m, __builtin_bit_cast(v2u16, p.w[j] & 0x7fff7fffu));
        const uint16_t most = m[0] > m[1] ? m[0] : m[1];
        if constexpr (std::is_same<T, bf16_t>::value) return (uint32_t)most << 16;
        else return __float_as_uint((float)__builtin_bit_cast(f16_t, most));
    }
}
__device__ __forceinline__ uint32_t most_of4lanes(uint32_t m) {
    uint32_t o = (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xB1, 15, 15, true);  // lane ^ 1
    m = o > m ? o : m;
    o = (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4E, 15, 15, true);  // lane ^ 2
    return o > m ? o : m;
}
constexpr uint32_t kInfBits = 0x7f800000u;

// The 8-bit checkpoint: value = code * 2^(scale - 133), scale the biased exponent of the block's largest magnitude; 255 stands for
// NaNs (a block that holds a NaN or an infinity).
__device__ __forceinline__ uint32_t ckpt8_scale(uint32_t most) { return most >= kInfBits ? 255u : most >> 23; }
// eight codes, round to nearest even, at most 127 (values from 127.5 steps on give up half a step: -128 and 128 are no codes)
__device__ __forceinline__ v2u ckpt8_codes(const float (&v)[8], uint32_t scale) {
    uint32_t t[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float q = __builtin_amdgcn_fmed3f(__builtin_amdgcn_ldexpf(v[j], 133 - (int)scale), -127.0f, 127.0f);
        t[j] = __float_as_uint(q + 12582912.0f);  // 1.5 * 2^23: rounds to the even integer and leaves it in the low byte
    }
    auto four = [](uint32_t a, uint32_t b, uint32_t c, uint32_t d) __attribute__((always_inline)) {
        return __builtin_amdgcn_perm(b, a, 0x0c0c0400u) | __builtin_amdgcn_perm(d, c, 0x04000c0cu);
    };
    return v2u{four(t[0], t[1], t[2], t[3]), four(t[4], t[5], t[6], t[7])};
}
// what one code step stands for, 2^(scale - 133); a NaN for 255
__device__ __forceinline__ float ckpt8_step(uint32_t scale) {
    const float s = __builtin_amdgcn_ldexpf(1.0f, (int)scale - 133);
    return scale == 255 ? __uint_as_float(0x7fc00000u) : s;
}
__device__ __forceinline__ void ckpt8_values(v2u c, float step, float (&v)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (float)(int8_t)(c[j / 4] >> (8 * (j & 3))) * step;
}

// Microscaled 4-bit floats (1 sign, 2 exponent and 1 mantissa bits: 0, .5, 1, 1.5, 2, 3, 4, 6): value = element * 2^(scale - 127),
// the largest element's exponent being that of the block's largest magnitude; 255 stands for NaNs.
__device__ __forceinline__ uint32_t mx4_scale(uint32_t most) {
    const uint32_t e = most >> 23;
    return most >= kInfBits ? 255u : e > 2 ? e - 2 : 0u;
}
// 2^(scale - 127); a NaN for 255
__device__ __forceinline__ float mx4_step(uint32_t scale) { return __uint_as_float(scale == 255 ? 0x7fc00000u : scale ? scale << 23 : 0x00400000u); }
// Eight codes, the first value in the lowest half byte.  The hardware's conversions divide by the scale, round to nearest even and
// saturate at 6, denormals included (compared with the definition over ties, edges and all three types).
template <class T>
__device__ __forceinline__ uint32_t mx4_codes(const Piece<T>& p, uint32_t scale) {
    const float s = __uint_as_float(scale ? scale << 23 : 0x00400000u);
    uint32_t c = 0;
    auto two = [&](int j) __attribute__((always_inline)) {
        if constexpr (std::is_same<T, float>::value) return v2f32{__uint_as_float(p.w[2 * j]), __uint_as_float(p.w[2 * j + 1])};
        else if constexpr (std::is_same<T, bf16_t>::value) return __builtin_bit_cast(v2bf16, p.w[j]);
        else return __builtin_bit_cast(v2f16, p.w[j]);
    };
    if constexpr (std::is_same<T, float>::value) {
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, two(0)[0], two(0)[1], s, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, two(1)[0], two(1)[1], s, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, two(2)[0], two(2)[1], s, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, two(3)[0], two(3)[1], s, 3);
    } else if constexpr (std::is_same<T, bf16_t>::value) {
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, two(0), s, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, two(1), s, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, two(2), s, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, two(3), s, 3);
    } else {
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, two(0), s, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, two(1), s, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, two(2), s, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, two(3), s, 3);
    }
    return scale == 255 ? 0 : c;
}

// ---- sums over groups of G = 16, 32 or 64 neighbouring lanes, the same value in every lane, without a trip through LDS
template <int G>
__device__ __forceinline__ float lanes_sum(float s) {
    auto step = [&](auto ctrl) __attribute__((always_inline)) {
        s += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(s), decltype(ctrl)::value, 15, 15, true));
    };
    step(std::integral_constant<int, 0xB1>());   // lane ^ 1
    step(std::integral_constant<int, 0x4E>());   // lane ^ 2
    step(std::integral_constant<int, 0x141>());  // the other four of eight
    step(std::integral_constant<int, 0x140>());  // the other eight of 16
    if constexpr (G >= 32) {
        const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(s), __float_as_uint(s), false, false);
        s = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    }
    if constexpr (G >= 64) {
        const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(s), __float_as_uint(s), false, false);
        s = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    }
    return s;
}

}  // namespace aq
