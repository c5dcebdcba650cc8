// The gradients of a fully connected layer from what it keeps in few bits:
//   weight gradient  dw[n][k] = sum_row dy[row][n] x8[row][k]      x8: the 8-bit checkpoint of its input
//   input gradient   dx[row][k] = sum_n dy[row][n] w4[n][k]        w4: its microscaled 4-bit weights
// Both are C[m][c] = sum_t A[m][t] B[t][c] on the bf16 matrix cores, without a rounding in front of the sums: a code of
// either format times its power of two has at most seven significant bits, so it is a bf16 value, and a value of dy is the sum of
// one (bfloat16), two (binary16) or three (fp32) bf16 values.
//
// A workgroup's 64 t of both operands go through LDS.  B lies there as it does in memory, t by t (and so does A for the weight
// gradient), and is transposed on its way to the registers: ds_read_b64_tr_b16 hands lane i of 16 the four t of column i out of
// four rows of 16 columns.
#include "learner.hpp"
#include "learner_device.hpp"

namespace aq {
namespace {

typedef short v4s16 __attribute__((ext_vector_type(4)));
typedef short v8s16 __attribute__((ext_vector_type(8)));

template <class T>
constexpr int kParts = std::is_same<T, float>::value ? 3 : std::is_same<T, f16_t>::value ? 2 : 1;

// Eight values as P bf16 parts, each the rest of the one before cut to bf16 (cut, not rounded: no part overflows, and three times
// eight bits are fp32's 24).  What is not finite is whole in the first.
template <class T, int P>
__device__ __forceinline__ void split(const Piece<T>& in, v4u (&out)[P]) {
    if constexpr (P == 1) {
        out[0] = v4u{in.w[0], in.w[1], in.w[2], in.w[3]};
    } else {
        float v[8];
        in.get(v);
#pragma unroll
        for (int q = 0; q < P; ++q) {
            uint32_t b[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                b[j] = __float_as_uint(v[j]) & 0xffff0000u;
                const bool finite = (__float_as_uint(v[j]) & 0x7fffffffu) < kInfBits;
                if (!finite && v[j] != v[j]) b[j] |= 0x00400000u;  // (a NaN stays one)
                v[j] = finite ? v[j] - __uint_as_float(b[j]) : 0.0f;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) out[q][j] = (b[2 * j] >> 16) | b[2 * j + 1];
        }
    }
}

// ---- LDS tiles
// [64 t][S columns]: 32-byte pieces of a row, piece p of row t in place p ^ turned(t), so that the 16 rows of a transposing
// read lie in different banks
__device__ __forceinline__ int turned(int t) { return (t & 3) | ((t >> 3) & 1) << 2; }
template <int S>
__device__ __forceinline__ int t_at(int t, int col) {  // byte address of column col (a multiple of 8) of row t
    return t * 2 * S + (((col >> 4) ^ (turned(t) & (S / 16 - 1))) << 5) + ((col & 8) << 1);
}
// 16 columns from col on, 32 t from t0 on, as an MFMA operand: lane l has column l mod 16, t = 8 (l / 16) .. + 7
template <int S>
__device__ __forceinline__ v8bf16 t_operand(const uint8_t* tile, int t0, int col, int lane) {
    typedef __attribute__((address_space(3))) v4s16* lds_ptr;
    const int g = lane >> 4, i = lane & 15, t = t0 + 8 * g + (i >> 2);
    const uint8_t* p = tile + t * 2 * S + (((col >> 4) ^ (turned(t) & (S / 16 - 1))) << 5) + (i & 3) * 8;
    const v4s16 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)p);
    const v4s16 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p + 4 * 2 * S));
    return __builtin_bit_cast(v8bf16, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}
// [S rows][64 t]: 16-byte pieces, piece p of row m in place p ^ (m / 2 mod 8)
__device__ __forceinline__ int m_at(int m, int piece) { return m * 128 + ((piece ^ ((m >> 1) & 7)) << 4); }

// ---- the operands.  Each thread fetches its part of 64 t into registers and later puts it into LDS as bf16.
// dy with t along the rows (weight gradient): [t][m]
template <class T, int S>
struct DyRows {
    static constexpr int P = kParts<T>, kUnits = S / 32, kPlane = 64 * 2 * S;
    static constexpr bool kTransposed = true;
    const T* d;
    int64_t ld;
    Piece<T> in[kUnits];
    __device__ __forceinline__ void fetch(int64_t t0, int64_t tn, int64_t m0, int64_t mn) {
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
            const int u = threadIdx.x + 256 * i;
            const int64_t t = t0 + u / (S / 8), m = m0 + 8 * (u % (S / 8));
            in[i].zero();
            if (t < tn) in[i].load(d + t * ld + m, (int)(mn - m < 8 ? mn - m : 8));
        }
    }
    __device__ __forceinline__ void put(uint8_t* to) const {
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
            const int u = threadIdx.x + 256 * i;
            v4u q[P];
            split<T, P>(in[i], q);
#pragma unroll
            for (int p = 0; p < P; ++p) *(v4u*)(to + p * kPlane + t_at<S>(u / (S / 8), 8 * (u % (S / 8)))) = q[p];
        }
    }
    static __device__ __forceinline__ v8bf16 operand(const uint8_t* tile, int t0, int m, int lane) { return t_operand<S>(tile, t0, m, lane); }
};
// dy with t along the columns (input gradient): [m][t]
template <class T, int S>
struct DyCols {
    static constexpr int P = kParts<T>, kUnits = S / 32, kPlane = 64 * 2 * S;
    static constexpr bool kTransposed = false;
    const T* d;
    int64_t ld;
    Piece<T> in[kUnits];
    __device__ __forceinline__ void fetch(int64_t t0, int64_t tn, int64_t m0, int64_t mn) {
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
            const int u = threadIdx.x + 256 * i;
            const int64_t m = m0 + u / 8, t = t0 + 8 * (u % 8);
            in[i].zero();
            if (m < mn) in[i].load(d + m * ld + t, (int)(tn - t < 8 ? tn - t : 8));
        }
    }
    __device__ __forceinline__ void put(uint8_t* to) const {
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
            const int u = threadIdx.x + 256 * i;
            v4u q[P];
            split<T, P>(in[i], q);
#pragma unroll
            for (int p = 0; p < P; ++p) *(v4u*)(to + p * kPlane + m_at(u / 8, u % 8)) = q[p];
        }
    }
    static __device__ __forceinline__ v8bf16 operand(const uint8_t* tile, int t0, int m, int lane) {
        return *(const v8bf16*)(tile + m_at(m + (lane & 15), t0 / 8 + (lane >> 4)));
    }
};
// checkpoint rows: 16 codes and a scale to a unit
template <int S>
struct KeptRows {
    static constexpr int kUnits = S / 64, kPlane = 64 * 2 * S;
    const uint8_t* codes;
    const uint8_t* scales;
    int64_t blocks;
    v4u c[kUnits];
    uint32_t s[kUnits];
    __device__ __forceinline__ void fetch(int64_t t0, int64_t tn, int64_t c0) {
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
            const int u = threadIdx.x + 256 * i;
            const int64_t t = t0 + u / (S / 16), b = (c0 + 16 * (u % (S / 16))) >> 5;
            c[i] = v4u{0, 0, 0, 0};
            s[i] = 0;
            if (t < tn && b < blocks) {
                c[i] = *(const v4u AQ_GLOBAL*)(codes + t * blocks * 32 + c0 + 16 * (u % (S / 16)));
                s[i] = ((const uint8_t AQ_GLOBAL*)scales)[t * blocks + b];
            }
        }
    }
    __device__ __forceinline__ void put(uint8_t* to) const {
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
            const int u = threadIdx.x + 256 * i, t = u / (S / 16), col = 16 * (u % (S / 16));
            const float step = ckpt8_step(s[i]);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float v[8];
                ckpt8_values(v2u{c[i][2 * h], c[i][2 * h + 1]}, step, v);
                Piece<bf16_t> o;
                o.set(v);
                *(v4u*)(to + t_at<S>(t, col + 8 * h)) = v4u{o.w[0], o.w[1], o.w[2], o.w[3]};
            }
        }
    }
};
// rows of 4-bit weights: a block of 32 to a unit
template <int S>
struct Mx4Rows {
    static constexpr int kUnits = S / 128 ? S / 128 : 1, kPlane = 64 * 2 * S;
    const uint8_t* codes;
    const uint8_t* scales;
    int64_t blocks;
    v4u c[kUnits];
    uint32_t s[kUnits];
    static __device__ __forceinline__ bool mine(int u) { return u < 64 * (S / 32); }
    __device__ __forceinline__ void fetch(int64_t t0, int64_t tn, int64_t c0) {
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
            const int u = threadIdx.x + 256 * i;
            const int64_t t = t0 + u / (S / 32), b = (c0 >> 5) + u % (S / 32);
            c[i] = v4u{0, 0, 0, 0};
            s[i] = 0;
            if (mine(u) && t < tn && b < blocks) {
                c[i] = *(const v4u AQ_GLOBAL*)(codes + (t * blocks + b) * 16);
                s[i] = ((const uint8_t AQ_GLOBAL*)scales)[t * blocks + b];
            }
        }
    }
    __device__ __forceinline__ void put(uint8_t* to) const {
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
            const int u = threadIdx.x + 256 * i, t = u / (S / 32), col = 32 * (u % (S / 32));
            if (!mine(u)) continue;
            const float step = mx4_step(s[i]);
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                v4u o;
                o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[i][h], step, 0));
                o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[i][h], step, 1));
                o[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[i][h], step, 2));
                o[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[i][h], step, 3));
                *(v4u*)(to + t_at<S>(t, col + 8 * h)) = o;
            }
        }
    }
};

// C tile of S x S, four wavefronts of S/2 x S/2.  blockIdx.z takes chunks [z * chunks, + chunks) of 64 t and writes its own C (and its
// own sums of A over t, where `sums` is given).
template <class A, class B, class T, int S>
__global__ void __launch_bounds__(256)
    k_grad(A a, B b, T* __restrict__ out, int64_t ld, int64_t out_stride, float* __restrict__ sums, int64_t mn, int64_t cn, int64_t tn,
           int chunks) {
    constexpr int P = A::P, H = S / 2, N = H / 16, kBuf = P * A::kPlane + B::kPlane;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t m0 = (int64_t)blockIdx.x * S, c0 = (int64_t)blockIdx.y * S;
    const int wm = (wave & 1) * H, wc = (wave >> 1) * H;
    int64_t t = (int64_t)blockIdx.z * chunks * 64;
    if (t + (int64_t)chunks * 64 < tn) tn = t + (int64_t)chunks * 64;
    const bool summing = sums && blockIdx.y == 0;
    float total[8];
    auto add = [&]() __attribute__((always_inline)) {
        if constexpr (A::kTransposed) {
            if (summing) {
#pragma unroll
                for (int i = 0; i < A::kUnits; ++i) {
                    float v[8];
                    a.in[i].get(v);
#pragma unroll
                    for (int j = 0; j < 8; ++j) total[j] += v[j];
                }
            }
        }
    };
#pragma unroll
    for (int j = 0; j < 8; ++j) total[j] = 0.0f;
    v4f32 acc[N][N];
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) acc[i][j] = v4f32{0, 0, 0, 0};
    a.fetch(t, tn, m0, mn);
    b.fetch(t, tn, c0);
    a.put(lds);
    b.put(lds + P * A::kPlane);
    add();
    __syncthreads();
    int buf = 0;
    for (; t < tn; t += 64) {
        const bool more = t + 64 < tn;
        if (more) {
            a.fetch(t + 64, tn, m0, mn);
            b.fetch(t + 64, tn, c0);
        }
        const uint8_t* const ta = lds + buf * kBuf;
        const uint8_t* const tb = ta + P * A::kPlane;
#pragma unroll
        for (int k = 0; k < 64; k += 32) {
            v8bf16 ob[N];
#pragma unroll
            for (int j = 0; j < N; ++j) ob[j] = t_operand<S>(tb, k, wc + 16 * j, lane);
#pragma unroll
            for (int p = P - 1; p >= 0; --p) {  // the smallest terms first
                v8bf16 oa[N];
#pragma unroll
                for (int i = 0; i < N; ++i) oa[i] = A::operand(ta + p * A::kPlane, k, wm + 16 * i, lane);
#pragma unroll
                for (int i = 0; i < N; ++i)
#pragma unroll
                    for (int j = 0; j < N; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ob[j], oa[i], acc[i][j], 0, 0, 0);
            }
        }
        buf ^= 1;
        if (more) {
            a.put(lds + buf * kBuf);
            b.put(lds + buf * kBuf + P * A::kPlane);
            add();
        }
        __syncthreads();
    }
    out += blockIdx.z * out_stride;
    const int r = lane & 15, g = lane >> 4;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int64_t m = m0 + wm + 16 * i + r;
        if (m >= mn) continue;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int64_t c = c0 + wc + 16 * j + 4 * g;
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = acc[i][j][e];
            if (c < cn) store4(out + m * ld, c, cn, v);
        }
    }
    if constexpr (A::kTransposed) {
        if (summing) {  // 256 / (S / 8) threads have a piece of eight columns each
            float* const red = (float*)lds;
#pragma unroll
            for (int j = 0; j < 8; ++j) red[(threadIdx.x / (S / 8)) * S + 8 * (threadIdx.x % (S / 8)) + j] = total[j];
            __syncthreads();
            if (threadIdx.x < S && m0 + threadIdx.x < mn) {
                float s = 0.0f;
#pragma unroll
                for (int i = 0; i < 2048 / S; ++i) s += red[i * S + threadIdx.x];
                sums[blockIdx.z * mn + m0 + threadIdx.x] = s;
            }
        }
    }
}

// the slices' results join, in their order: dw, and dy's sums behind it
__global__ void __launch_bounds__(256) k_grad_join(const float* __restrict__ part, int slices, int64_t m, int64_t c, float* __restrict__ out,
                                                   int64_t ld, const float* __restrict__ part_sums, float* __restrict__ sums) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i < m * c) {
        float s = 0.0f;
        for (int k = 0; k < slices; ++k) s += part[k * m * c + i];
        out[i / c * ld + i % c] = s;
    } else if (sums && i < m * c + m) {
        float s = 0.0f;
        for (int k = 0; k < slices; ++k) s += part_sums[k * m + (i - m * c)];
        sums[i - m * c] = s;
    }
}

// how a product of m x c over t runs: tiles of S x S, z slices of t
struct Plan {
    int s, z, chunks;
};
Plan plan(int64_t m, int64_t c, int64_t t, bool split_t) {
    auto tiles = [&](int64_t s) { return ((m + s - 1) / s) * ((c + s - 1) / s); };
    Plan p;
    p.s = 128;
    const int64_t all = (t + 63) / 64;
    int64_t z = 1;
    if (split_t) {
        z = 512 / tiles(p.s);
        if (z > all / 4) z = all / 4;
        if (z < 1) z = 1;
    } else if (tiles(128) < 256) {
        p.s = 64;
    }
    p.chunks = (int)((all + z - 1) / z);
    p.z = p.chunks ? (int)((all + p.chunks - 1) / p.chunks) : 1;
    return p;
}

template <class A, class B, class T, int S>
aq_status launch(const A& a, const B& b, T* out, int64_t ld, int64_t stride, float* sums, int64_t m, int64_t c, int64_t t, const Plan& p,
                 hipStream_t st) {
    constexpr int kLds = 2 * (A::P * A::kPlane + B::kPlane);
    auto* const k = k_grad<A, B, T, S>;
    if (hip_failed(hipFuncSetAttribute((const void*)k, hipFuncAttributeMaxDynamicSharedMemorySize, kLds))) return AQ_EHIP;
    k<<<dim3((unsigned)((m + S - 1) / S), (unsigned)((c + S - 1) / S), (unsigned)p.z), 256, kLds, st>>>(a, b, out, ld, stride, sums, m, c, t, p.chunks);
    return hip_failed(hipGetLastError()) ? AQ_EHIP : AQ_OK;
}

}  // namespace

int64_t weight_grad_workspace(int64_t rows, int64_t n, int64_t k) {
    const Plan p = plan(n, k, rows, true);
    return p.z > 1 ? p.z * (n * k + n) * (int64_t)sizeof(float) : 0;
}

aq_status launch_weight_grad(const aq_matrix& dy, const aq_ckpt8& kept, const aq_matrix& dw, float* db, void* ws, hipStream_t st) {
    const int64_t n = dy.cols, k = kept.cols, rows = dy.rows;
    const Plan p = plan(n, k, rows, true);
    const bool join = p.z > 1;
    float* const out = join ? (float*)ws : (float*)dw.d;
    float* const sums = !db ? nullptr : join ? (float*)ws + p.z * n * k : db;
    const aq_status s = with_dtype(dy.dtype, [&](auto t) {
        using T = decltype(t);
        constexpr int S = 128;
        return launch<DyRows<T, S>, KeptRows<S>, float, S>({(const T*)dy.d, dy.ld}, {(const uint8_t*)kept.d_codes, kept.d_scales, blocks32(k)}, out,
                                                           join ? k : dw.ld, n * k, sums, n, k, rows, p, st);
    });
    if (s != AQ_OK || !join) return s;
    k_grad_join<<<(unsigned)((n * k + n + 255) / 256), 256, 0, st>>>((const float*)ws, p.z, n, k, (float*)dw.d, dw.ld, sums, db);
    return hip_failed(hipGetLastError()) ? AQ_EHIP : AQ_OK;
}

int64_t input_grad_workspace(int64_t rows, int64_t n, int64_t k) { return 0; }

aq_status launch_input_grad(const aq_matrix& dy, const aq_mx4& w, const aq_matrix& dx, void* ws, hipStream_t st) {
    const int64_t n = w.rows, k = w.cols, rows = dy.rows;
    const Plan p = plan(rows, k, n, false);
    return with_dtype(dy.dtype, [&](auto t) {
        using T = decltype(t);
        auto go = [&](auto sc) {
            constexpr int S = decltype(sc)::value;
            return launch<DyCols<T, S>, Mx4Rows<S>, T, S>({(const T*)dy.d, dy.ld}, {(const uint8_t*)w.d_codes, w.d_scales, blocks32(k)}, (T*)dx.d,
                                                          dx.ld, 0, nullptr, rows, k, n, p, st);
        };
        return p.s == 64 ? go(std::integral_constant<int, 64>()) : go(std::integral_constant<int, 128>());
    });
}

}  // namespace aq
