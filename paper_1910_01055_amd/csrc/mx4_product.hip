// Products of microscaled 4-bit matrices on the scaled matrix cores: y[m][n] = sum_k x[m][k] w[n][k] + bias[n].
//
// A block of 32 values is 16 bytes and one scale, which is what one lane of the scaled MFMA holds of one row: operands go from
// memory to the matrix cores as they lie.  v_mfma_scale_f32_16x16x128: lane l holds row l mod 16, block l / 16 of four;
// v_mfma_scale_f32_32x32x64: row l mod 32, block l / 32 of two.  The weights are the first operand, so that a lane ends up with
// four neighbouring features of one row of y.
#include "learner.hpp"
#include "learner_device.hpp"

namespace aq {
namespace {

typedef int v8i32 __attribute__((ext_vector_type(8)));
typedef float v16f32 __attribute__((ext_vector_type(16)));
constexpr int kFp4 = 4;  // the instructions' number of the 4-bit format

__device__ __forceinline__ v8i32 operand(v4u c) { return v8i32{(int)c[0], (int)c[1], (int)c[2], (int)c[3], 0, 0, 0, 0}; }

// ---- few rows: 16 features to a workgroup, whose W wavefronts take turns along k and join their sums in LDS; RT tiles of 16 rows.
struct Blocks {  // rows that are quantized already
    const uint8_t* codes;
    const uint8_t* scales;
    int64_t blocks;
    __device__ __forceinline__ void get(int64_t row, int64_t b, v4u& c, uint32_t& scale) const {
        c = *(const v4u AQ_GLOBAL*)(codes + (row * blocks + b) * 16);
        scale = ((const uint8_t AQ_GLOBAL*)scales)[row * blocks + b];
    }
};
template <class T>
struct Values {  // rows of values, quantized in the lane that needs them
    const T* x;
    int64_t ld;
    int cols;
    __device__ __forceinline__ void get(int64_t row, int64_t b, v4u& c, uint32_t& scale) const {
        const T* p = x + row * ld + b * 32;
        const int n = cols - (int)b * 32;
        Piece<T> q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i].load(p + 8 * i, n - 8 * i);
        float v[4][8];
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            q[i].get(v[i]);
            const uint32_t m = most_of8(v[i]);
            most = m > most ? m : most;
        }
        scale = mx4_scale(most);
#pragma unroll
        for (int i = 0; i < 4; ++i) c[i] = mx4_codes(v[i], scale);
    }
};

template <class X, class T, int RT, int W>
__global__ void __launch_bounds__(64 * W)
    k_mx4_rows(X x, Blocks w, const float* __restrict__ bias, T* __restrict__ y, int64_t ldy, int rows, int n, int blocks) {
    __shared__ v4f32 part[W][RT][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
    const int64_t n0 = (int64_t)blockIdx.x * 16, m0 = (int64_t)blockIdx.y * (16 * RT);
    v4f32 acc[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) acc[i] = v4f32{0, 0, 0, 0};
    for (int b0 = 4 * wave; b0 < blocks; b0 += 4 * W) {
        const int b = b0 + g;
        v4u cw{0, 0, 0, 0}, cx[RT];
        uint32_t sw = 0, sx[RT];
        if (b < blocks && n0 + r < n) w.get(n0 + r, b, cw, sw);
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            cx[i] = v4u{0, 0, 0, 0};
            sx[i] = 0;
            if (b < blocks && m0 + 16 * i + r < rows) x.get(m0 + 16 * i + r, b, cx[i], sx[i]);
        }
#pragma unroll
        for (int i = 0; i < RT; ++i)
            acc[i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(cw), operand(cx[i]), acc[i], kFp4, kFp4, 0, (int)sw, 0, (int)sx[i]);
    }
#pragma unroll
    for (int i = 0; i < RT; ++i) part[wave][i][lane] = acc[i];
    __syncthreads();
    for (int i = wave; i < RT; i += W) {
        v4f32 s = part[0][i][lane];
#pragma unroll
        for (int j = 1; j < W; ++j) s += part[j][i][lane];
        const int64_t row = m0 + 16 * i + r, f = n0 + 4 * g;
        if (row < rows && f < n) {
            float v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = s[j] + (bias && f + j < n ? bias[f + j] : 0.0f);
            store4(y + row * ldy, f, n, v);
        }
    }
}

// ---- many rows: BM rows x BN features to a workgroup of four wavefronts (2 x 2), 256 k at a time through LDS.  A chunk of a row
// is 128 bytes; its 16-byte block s lies in place s ^ (row / 2 mod 8), so that the 16 rows which a read takes at once lie in
// different banks.
template <class T, int BM, int BN>
__global__ void __launch_bounds__(256, 1)
    k_mx4_tiles(Blocks x, Blocks w, const float* __restrict__ bias, T* __restrict__ y, int64_t ldy, int rows, int n, int blocks) {
    constexpr int R = BM + BN, U = R / 32, SU = (R + 255) / 256, TM = BM / 64, TN = BN / 64;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];  // two buffers: [R][128] codes, [R][8] scales
    constexpr int kBuf = R * 136;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = lane & 31, g = lane >> 5;
    const int64_t m0 = (int64_t)blockIdx.x * BM, n0 = (int64_t)blockIdx.y * BN;
    const int wm = (wave & 1) * (BM / 2), wn = (wave >> 1) * (BN / 2);
    v4u c[U];
    v2u s[SU];
    auto fetch = [&](int b0) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int u = tid + 256 * i, row = u >> 3, b = b0 + (u & 7);
            const bool is_x = i < BM / 32;  // (rows of x first)
            const int64_t at = is_x ? m0 + row : n0 + row - BM;
            c[i] = v4u{0, 0, 0, 0};
            if (b < blocks && at < (is_x ? rows : n)) c[i] = *(const v4u AQ_GLOBAL*)((is_x ? x.codes : w.codes) + (at * blocks + b) * 16);
        }
#pragma unroll
        for (int i = 0; i < SU; ++i) {
            const int row = tid + 256 * i;
            const bool is_x = row < BM;
            const int64_t at = is_x ? m0 + row : n0 + row - BM;
            s[i] = v2u{0, 0};
            if (row < R && at < (is_x ? rows : n)) {
                const uint8_t* p = (is_x ? x.scales : w.scales) + at * blocks + b0;
                if (b0 + 8 <= blocks) {
                    typedef v2u v2u_byte __attribute__((aligned(1)));
                    s[i] = *(const v2u_byte AQ_GLOBAL*)p;
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (b0 + j < blocks) s[i][j / 4] |= (uint32_t)p[j] << (8 * (j & 3));
                }
            }
        }
    };
    auto put = [&](uint8_t* to) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int u = tid + 256 * i, row = u >> 3;
            *(v4u*)(to + row * 128 + (((u & 7) ^ ((row >> 1) & 7)) << 4)) = c[i];
        }
#pragma unroll
        for (int i = 0; i < SU; ++i)
            if (tid + 256 * i < R) *(v2u*)(to + R * 128 + (tid + 256 * i) * 8) = s[i];
    };
    v16f32 acc[TN][TM];
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
    fetch(0);
    put(lds);
    __syncthreads();
    int buf = 0;
    for (int b0 = 0; b0 < blocks; b0 += 8) {
        const bool more = b0 + 8 < blocks;
        if (more) fetch(b0 + 8);
        const uint8_t* from = lds + buf * kBuf;
        v2u sx[TM], sw[TN];
#pragma unroll
        for (int j = 0; j < TM; ++j) {
            sx[j] = *(const v2u*)(from + R * 128 + (wm + 32 * j + r) * 8);
            sx[j] = v2u{sx[j][0] >> (8 * g), sx[j][1] >> (8 * g)};
        }
#pragma unroll
        for (int i = 0; i < TN; ++i) {
            sw[i] = *(const v2u*)(from + R * 128 + (BM + wn + 32 * i + r) * 8);
            sw[i] = v2u{sw[i][0] >> (8 * g), sw[i][1] >> (8 * g)};
        }
        auto turn = [&](auto k) __attribute__((always_inline)) {
            constexpr int K = decltype(k)::value;  // 64 of the chunk's 256
            v4u cx[TM], cw[TN];
#pragma unroll
            for (int j = 0; j < TM; ++j) {
                const int row = wm + 32 * j + r;
                cx[j] = *(const v4u*)(from + row * 128 + (((2 * K + g) ^ ((row >> 1) & 7)) << 4));
            }
#pragma unroll
            for (int i = 0; i < TN; ++i) {
                const int row = BM + wn + 32 * i + r;
                cw[i] = *(const v4u*)(from + row * 128 + (((2 * K + g) ^ ((row >> 1) & 7)) << 4));
            }
#pragma unroll
            for (int i = 0; i < TN; ++i)
#pragma unroll
                for (int j = 0; j < TM; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(cw[i]), operand(cx[j]), acc[i][j], kFp4, kFp4, 2 * (K & 1),
                                                                            (int)sw[i][K / 2], 2 * (K & 1), (int)sx[j][K / 2]);
        };
        turn(std::integral_constant<int, 0>());
        turn(std::integral_constant<int, 1>());
        turn(std::integral_constant<int, 2>());
        turn(std::integral_constant<int, 3>());
        buf ^= 1;
        if (more) put(lds + buf * kBuf);
        __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < TM; ++j) {
        const int64_t row = m0 + wm + 32 * j + r;
        if (row >= rows) continue;
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int64_t f = n0 + wn + 32 * i + 8 * q + 4 * g;
                if (f >= n) continue;
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = acc[i][j][4 * q + e] + (bias && f + e < n ? bias[f + e] : 0.0f);
                store4(y + row * ldy, f, n, v);
            }
    }
}

Blocks blocks_of(const aq_mx4& q) { return {(const uint8_t*)q.d_codes, q.d_scales, blocks32(q.cols)}; }

constexpr int64_t kFewRows = 64;

template <class X, class T>
aq_status launch_rows(const X& x, int64_t rows, const aq_mx4& w, const float* bias, const aq_matrix& y, hipStream_t st) {
    const dim3 grid((unsigned)((w.rows + 15) / 16), (unsigned)((rows + 15) / 16));
    k_mx4_rows<X, T, 1, 8><<<grid, 512, 0, st>>>(x, blocks_of(w), bias, (T*)y.d, y.ld, (int)rows, (int)w.rows, (int)blocks32(w.cols));
    return hip_failed(hipGetLastError()) ? AQ_EHIP : AQ_OK;
}

template <class T>
aq_status launch_tiles(const aq_mx4& x, const aq_mx4& w, const float* bias, const aq_matrix& y, hipStream_t st) {
    constexpr int BM = 128, BN = 128, kLds = 2 * (BM + BN) * 136;
    auto* const k = k_mx4_tiles<T, BM, BN>;
    if (hip_failed(hipFuncSetAttribute((const void*)k, hipFuncAttributeMaxDynamicSharedMemorySize, kLds))) return AQ_EHIP;
    const dim3 grid((unsigned)((x.rows + BM - 1) / BM), (unsigned)((w.rows + BN - 1) / BN));
    k<<<grid, 256, kLds, st>>>(blocks_of(x), blocks_of(w), bias, (T*)y.d, y.ld, (int)x.rows, (int)w.rows, (int)blocks32(w.cols));
    return hip_failed(hipGetLastError()) ? AQ_EHIP : AQ_OK;
}

}  // namespace

int64_t mx4_linear_workspace(int64_t rows, int64_t n, int64_t k) {
    if (rows <= kFewRows) return 0;
    const int64_t b = rows * blocks32(k);
    return 16 * b + (b + 15) / 16 * 16;
}

aq_status launch_mx4_matmul(const aq_mx4& x, const aq_mx4& w, const float* bias, const aq_matrix& y, hipStream_t st) {
    return with_dtype(y.dtype, [&](auto t) {
        using T = decltype(t);
        if (x.rows <= kFewRows) return launch_rows<Blocks, T>(blocks_of(x), x.rows, w, bias, y, st);
        return launch_tiles<T>(x, w, bias, y, st);
    });
}

aq_status launch_mx4_linear(const aq_matrix& x, const aq_mx4& w, const float* bias, const aq_matrix& y, void* ws, hipStream_t st) {
    if (x.rows <= kFewRows)
        return with_dtype(x.dtype, [&](auto t) {
            using T = decltype(t);
            return launch_rows<Values<T>, T>(Values<T>{(const T*)x.d, x.ld, (int)x.cols}, x.rows, w, bias, y, st);
        });
    const int64_t b = x.rows * blocks32(x.cols);
    const aq_mx4 q = {ws, (uint8_t*)ws + 16 * b, x.rows, x.cols};
    const aq_status s = launch_mx4_quantize(x, q, st);
    return s != AQ_OK ? s : launch_mx4_matmul(q, w, bias, y, st);
}

}  // namespace aq
