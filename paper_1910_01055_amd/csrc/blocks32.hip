// The two block formats to and from rows of values: 8-bit checkpoints and microscaled 4-bit floats.
//
// Bound by memory (65536 x 2048 bfloat16 values to checkpoints: 70 us, 5.8 TB/s of reads and writes, and back 68, 6.0 TB/s; 16384 x 4096
// to 4-bit floats: 35 us, 4.8 TB/s).  A thread holds eight values, four neighbouring threads a block, whose largest magnitude they find by two
// exchanges within their quad; L = 4 .. 64 threads walk along a row (few, so that short rows share a wavefront), a workgroup
// takes 256 / L rows at a time.
#include "learner.hpp"
#include "learner_device.hpp"

namespace aq {
namespace {

constexpr int kThreads = 256;

struct Ckpt8 {
    static constexpr int kBits = 8;  // of a code
    template <class T>
    static __device__ __forceinline__ void pack(const Piece<T>& p, uint8_t* codes, uint32_t& scale) {
        scale = ckpt8_scale(most_of4lanes(most_of(p)));
        float v[8];
        p.get(v);
        *(v2u*)codes = ckpt8_codes(v, scale);
    }
    // four values
    typedef uint32_t Codes4;
    static __device__ __forceinline__ void unpack4(uint32_t c, uint32_t scale, float* v) {
        const float step = ckpt8_step(scale);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = (float)(int8_t)(c >> (8 * j)) * step;
    }
};
struct Mx4 {
    static constexpr int kBits = 4;
    template <class T>
    static __device__ __forceinline__ void pack(const Piece<T>& p, uint8_t* codes, uint32_t& scale) {
        scale = mx4_scale(most_of4lanes(most_of(p)));
        *(uint32_t*)codes = mx4_codes(p, scale);
    }
    typedef uint16_t Codes4;
    static __device__ __forceinline__ void unpack4(uint32_t c, uint32_t scale, float* v) {
        const float s = mx4_step(scale);
        const v2f32 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 1);
        v[0] = a[0];
        v[1] = a[1];
        v[2] = b[0];
        v[3] = b[1];
    }
};

template <class Format, class T, int L>
__global__ void __launch_bounds__(kThreads)
    k_to_blocks(const T* __restrict__ x, int64_t ld, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales, int rows, int cols, int blocks) {
    const int piece = blockIdx.x * L + threadIdx.x % L;
    if (piece >= 4 * blocks) return;  // (whole quads)
    const int64_t step = (int64_t)gridDim.y * (kThreads / L);
    for (int64_t row = (int64_t)blockIdx.y * (kThreads / L) + threadIdx.x / L; row < rows; row += step) {
        Piece<T> in;
        in.load(x + row * ld + 8 * (int64_t)piece, cols - 8 * piece);
        uint32_t scale;
        Format::pack(in, codes + (row * blocks * 4 + piece) * Format::kBits, scale);
        if ((threadIdx.x & 3) == 0) scales[row * blocks + (piece >> 2)] = (uint8_t)scale;
    }
}

// Stores of 16 bytes to a thread, so that a wavefront's lie side by side: V values of T (2048 x 2048 to fp32: 6.9 us with 32 bytes a
// thread in two stores, 5.7 in one).
template <class Format, class T, int L>
__global__ void __launch_bounds__(kThreads)
    k_from_blocks(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, T* __restrict__ x, int64_t ld, int rows, int cols,
                  int blocks) {
    constexpr int V = 16 / (int)sizeof(T);
    const int piece = blockIdx.x * L + threadIdx.x % L;
    const int left = cols - V * piece;
    if (left <= 0) return;
    const int64_t step = (int64_t)gridDim.y * (kThreads / L);
    for (int64_t row = (int64_t)blockIdx.y * (kThreads / L) + threadIdx.x / L; row < rows; row += step) {
        typedef typename Format::Codes4 C4;
        C4 c[V / 4];
        const uint32_t scale = scales[row * blocks + piece / (32 / V)];
        const C4* const from = (const C4*)(codes + (row * blocks * 32 + V * (int64_t)piece) * Format::kBits / 8);
#pragma unroll
        for (int i = 0; i < V / 4; ++i) c[i] = from[i];
        float v[8];
#pragma unroll
        for (int i = 0; i < V / 4; ++i) Format::unpack4(c[i], scale, v + 4 * i);
        T* const to = x + row * ld + V * (int64_t)piece;
        if constexpr (V == 4) {
            if (left >= 4) {
                *(v4u_any AQ_GLOBAL*)to = v4u{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
            } else {
#pragma unroll
                for (int j = 0; j < 3; ++j)
                    if (j < left) to[j] = v[j];
            }
        } else {
            Piece<T> out;
            out.set(v);
            out.store(to, left);
        }
    }
}

// calls go(L, grid) for rows of so many pieces
template <class Go>
aq_status by_width(int64_t rows, int64_t pieces, Go&& go) {
    auto with = [&](auto l) {
        constexpr int L = decltype(l)::value;
        const int64_t y = (rows + kThreads / L - 1) / (kThreads / L);
        go(l, dim3((unsigned)((pieces + L - 1) / L), (unsigned)(y < 65535 ? y : 65535)));
        return hip_failed(hipGetLastError()) ? AQ_EHIP : AQ_OK;
    };
    if (pieces <= 4) return with(std::integral_constant<int, 4>());
    if (pieces <= 8) return with(std::integral_constant<int, 8>());
    if (pieces <= 16) return with(std::integral_constant<int, 16>());
    if (pieces <= 32) return with(std::integral_constant<int, 32>());
    return with(std::integral_constant<int, 64>());
}

template <class Format>
aq_status to_blocks(const aq_matrix& x, void* codes, uint8_t* scales, hipStream_t st) {
    return with_dtype(x.dtype, [&](auto t) {
        using T = decltype(t);
        return by_width(x.rows, 4 * blocks32(x.cols), [&](auto l, dim3 grid) {
            k_to_blocks<Format, T, decltype(l)::value><<<grid, kThreads, 0, st>>>((const T*)x.d, x.ld, (uint8_t*)codes, scales, (int)x.rows,
                                                                                (int)x.cols, (int)blocks32(x.cols));
        });
    });
}
template <class Format>
aq_status from_blocks(const void* codes, const uint8_t* scales, const aq_matrix& x, hipStream_t st) {
    return with_dtype(x.dtype, [&](auto t) {
        using T = decltype(t);
        constexpr int V = 16 / (int)sizeof(T);
        return by_width(x.rows, (x.cols + V - 1) / V, [&](auto l, dim3 grid) {
            k_from_blocks<Format, T, decltype(l)::value><<<grid, kThreads, 0, st>>>((const uint8_t*)codes, scales, (T*)x.d, x.ld, (int)x.rows,
                                                                                  (int)x.cols, (int)blocks32(x.cols));
        });
    });
}

}  // namespace

aq_status launch_ckpt8_pack(const aq_matrix& x, const aq_ckpt8& kept, hipStream_t st) {
    return to_blocks<Ckpt8>(x, kept.d_codes, kept.d_scales, st);
}
aq_status launch_ckpt8_unpack(const aq_ckpt8& kept, const aq_matrix& x, hipStream_t st) {
    return from_blocks<Ckpt8>(kept.d_codes, kept.d_scales, x, st);
}
aq_status launch_mx4_quantize(const aq_matrix& x, const aq_mx4& q, hipStream_t st) { return to_blocks<Mx4>(x, q.d_codes, q.d_scales, st); }
aq_status launch_mx4_dequantize(const aq_mx4& q, const aq_matrix& x, hipStream_t st) { return from_blocks<Mx4>(q.d_codes, q.d_scales, x, st); }

}  // namespace aq
