// Products of microscaled 4-bit matrices on the scaled matrix cores: y[m][n] = sum_k x[m][k] w[n][k] + bias[n].
//
// A block of 32 values is 16 bytes and one scale, which is what one lane of the scaled MFMA holds of one row: operands go from
// memory to the matrix cores as they lie.  v_mfma_scale_f32_16x16x128: lane l holds row l mod 16, block l / 16 of four;
// v_mfma_scale_f32_32x32x64: row l mod 32, block l / 32 of two.  The weights are the first operand, so that a lane ends up with
// four neighbouring features of one row of y.
#include "learner.hpp"
#include "product_device.hpp"

namespace aq {
namespace {

typedef int v8i32 __attribute__((ext_vector_type(8)));
constexpr int kFp4 = 4;  // the instructions' number of the 4-bit format

__device__ __forceinline__ v8i32 operand(v4u c) { return v8i32{(int)c[0], (int)c[1], (int)c[2], (int)c[3], 0, 0, 0, 0}; }

// ---- few rows: 16 features by 16 rows to a workgroup, whose eight wavefronts take turns along k and join their sums in LDS.  Bound by
// latency: a launch, a trip to memory for every 1024 k, a barrier (2048 x 2048 weights, one bfloat16 row: 3.9 us, of which an empty
// kernel is 2.3, 16 rows 4.1; with four wavefronts 4.3 and 4.5, with the next turn requested before the present one's work 4.2 and 4.4, as
// fewer wavefronts fit).
// What 64 lanes need of 16 rows and four blocks of them: lane l the block l / 16 of row l mod 16.
struct Blocks {  // rows that are quantized already
    static constexpr int kLds = 0;
    const uint8_t* codes;
    const uint8_t* scales;
    int64_t blocks;
    struct Raw {
        v4u c;
        uint32_t scale;
    };
    // Rows from row0 on, of which `rows` exist, and blocks from b0 on; where there is none the last one, whose results are not stored or,
    // with zeros for x, add nothing (a NaN's block only to a row that is NaN).
    __device__ __forceinline__ void request(int row0, int rows, int b0, int lane, Raw& q) const {
        const int row = row0 + (lane & 15), b = b0 + (lane >> 4);
        const int64_t at = (row < rows ? row : rows - 1) * blocks + (b < blocks ? b : (int)blocks - 1);
        q.c = *(const v4u AQ_GLOBAL*)(codes + at * 16);
        q.scale = ((const uint8_t AQ_GLOBAL*)scales)[at];
    }
    __device__ __forceinline__ void get(const Raw& q, uint8_t*, int lane, int left, v4u& c, uint32_t& scale) const {
        c = lane >> 4 < left ? q.c : v4u{0, 0, 0, 0};
        scale = q.scale;
    }
};
// Rows of values, quantized here.  Four lanes load a block, so that they read whole lines (each lane a block of its own: 16 fp32 rows
// of 4096 into 4096 features 11.4 us for 6.1), lane l eight values of row l / 4; the codes change lanes in LDS.
template <class T>
struct Values {
    static constexpr int kLds = 1024;  // bytes of a wavefront's own
    const T* x;
    int64_t ld;
    int cols;
    struct Raw {
        Piece<T> q[4];
    };
    __device__ __forceinline__ void request(int row0, int rows, int b0, int lane, Raw& raw) const {
        const int row = row0 + (lane >> 2), col = 32 * b0 + 8 * (lane & 3);
        const T* const p = x + (row < rows ? row : rows - 1) * ld + col;
        if (32 * b0 + 128 <= cols) {
#pragma unroll
            for (int i = 0; i < 4; ++i) raw.q[i].load_all(p + 32 * i);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) raw.q[i].load(p + 32 * i, cols - col - 32 * i);
        }
    }
    __device__ __forceinline__ void get(const Raw& raw, uint8_t* lds, int lane, int, v4u& c, uint32_t& scale) const {
        uint32_t scales = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t s = mx4_scale(most_of4lanes(most_of(raw.q[i])));
            scales |= s << (8 * i);
            *(uint32_t*)(lds + 256 * i + 4 * lane) = mx4_codes(raw.q[i], s);
        }
        __builtin_amdgcn_wave_barrier();  // (a wavefront's accesses to LDS are done in their order)
        c = *(const v4u*)(lds + 16 * lane);
        scale = (uint32_t)__builtin_amdgcn_ds_bpermute(16 * (lane & 15), (int)scales) >> (8 * (lane >> 4));
        __builtin_amdgcn_wave_barrier();
    }
};

template <class X, class T>
__global__ void __launch_bounds__(512)
    k_mx4_rows(X x, Blocks w, const float* __restrict__ bias, T* __restrict__ y, int64_t ldy, int rows, int n, int blocks) {
    constexpr int W = 8;  // wavefronts
    __shared__ v4f32 part[W][64];
    static_assert(X::kLds <= sizeof(part[0]), "");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * 16, row0 = blockIdx.y * 16, row = row0 + r;
    v4f32 acc{0, 0, 0, 0};
    for (int b = 4 * wave; b < blocks; b += 4 * W) {
        typename Blocks::Raw own;
        typename X::Raw raw;
        w.request(n0, n, b, lane, own);
        x.request(row0, rows, b, lane, raw);
        v4u cx;
        uint32_t sx;
        x.get(raw, (uint8_t*)part[wave], lane, blocks - b, cx, sx);
        acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(own.c), operand(cx), acc, kFp4, kFp4, 0, (int)own.scale, 0, (int)sx);
    }
    part[wave][lane] = acc;
    __syncthreads();
    if (wave == 0) {
        v4f32 s = part[0][lane];
#pragma unroll
        for (int j = 1; j < W; ++j) s += part[j][lane];
        const int f = n0 + 4 * g;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (row < rows && f + j < n) y[row * ldy + f + j] = (T)(s[j] + (bias ? bias[f + j] : 0.0f));
    }
}

// ---- many rows: S rows x S features to a workgroup, a wavefront takes 32 TM rows and 32 TN features.  256 k of a row are 128 bytes, a
// chunk; its 16-byte block s lies in LDS in place s ^ (row / 2 mod 8), so that the 16 rows which a read takes at once lie in different
// banks.  Chunks go from memory to LDS by themselves (buffer loads to LDS, which fill it with zeros behind a matrix's end) into
// two buffers.  A chunk's products come in four turns of 64 k, whose operands are read a turn ahead; behind the third all of a
// chunk is in registers, and the barrier there hands its buffer to the chunk after the next.  Scales come for two chunks at a time
// through registers.
//
// 16384 x 4096 x 4096 to bfloat16: 160 us alone, 177 to 202 back to back (2.7 to 3.4 PFLOP/s), where a loop of nothing but these
// products on such values reaches 6.5 at the clock that is left.  Without the loads it would take 129, without the products 112: the two
// do not overlap wholly.  128 k at a time, half a line of memory to a row: 170; tiles of 128 x 128 to a wavefront, one to a SIMD: 186.
template <class T, int S, int NT>
__global__ void __launch_bounds__(NT, 1)
    k_mx4_tiles(Blocks x, Blocks w, const float* __restrict__ bias, T* __restrict__ y, int64_t ldy, int rows, int n, int blocks) {
    constexpr int R = 2 * S, SU = (R + NT - 1) / NT, J = R * 8 / NT, TM = S / 64, TN = S / (NT / 128) / 32, kBuf = R * 128;
    static_assert(NT / 64 * 32 * kOutRow<T, TN> <= 2 * kBuf, "results leave through the buffers");
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];  // two buffers of chunks; scales of four chunks
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 31, g = lane >> 5;
    const Place at = place_of_workgroup((uint32_t)((rows + S - 1) / S), (uint32_t)((n + S - 1) / S));
    const int64_t m0 = (int64_t)at.m * S, n0 = (int64_t)at.c * S, pitch = (int64_t)blocks * 16;
    const int wm = (wave & 1) * (S / 2), wn = S + (wave >> 1) * (32 * TN), chunks = (blocks + 7) / 8;
    Window win_x, win_w;
    win_x.set(x.codes, m0 * pitch, rows * pitch);
    win_w.set(w.codes, n0 * pitch, n * pitch);
    // unit j of a thread: row (tid + NT j) / 8 of both matrices' rows, place tid mod 8
    const int block = (tid & 7) ^ ((tid >> 4) & 7);
    int off[J];
#pragma unroll
    for (int j = 0; j < J; ++j) off[j] = (((tid + NT * j) >> 3) % S) * (int)pitch + block * 16;
    auto fetch = [&](int chunk) __attribute__((always_inline)) {
        const int from = 8 * chunk + block < blocks ? 128 * chunk : Window::kOutside;
#pragma unroll
        for (int j = 0; j < J; ++j)
            load_to_lds(j < J / 2 ? win_x : win_w, off[j] + from, lds + (chunk & 1) * kBuf + (wave * 64 + NT * j) * 16);
    };
    // a thread's rows of scales (some row that exists where it has none: what comes of it is not stored)
    auto clamp = [](int64_t row, int most) __attribute__((always_inline)) { return row < most ? row : (int64_t)most - 1; };
    const uint8_t* scale_row[SU];
    v4u sc[SU];
#pragma unroll
    for (int i = 0; i < SU; ++i) {
        const int row = (tid + NT * i) % R;
        scale_row[i] = row < S ? x.scales + clamp(m0 + row, rows) * blocks : w.scales + clamp(n0 + row - S, n) * blocks;
    }
    // Of blocks b0 .. b0 + 15.  Where a row ends before, its last 16 moved to where they belong, or as few as there are (byte by byte
    // 16384 x 4480 x 4096 204 us for 184, 4096 x 256 x 2048 9.2 for 8.6).
    auto fetch_scales = [&](int b0) __attribute__((always_inline)) {
        typedef v4u v4u_byte __attribute__((aligned(1)));
        typedef v2u v2u_byte __attribute__((aligned(1)));
        typedef uint32_t u32_byte __attribute__((aligned(1)));
        typedef uint16_t u16_byte __attribute__((aligned(1)));
        const int more = b0 + 16 - blocks;  // bytes of the last 16 in front of block b0
        if (more <= 0) {
#pragma unroll
            for (int i = 0; i < SU; ++i) sc[i] = *(const v4u_byte AQ_GLOBAL*)(scale_row[i] + b0);
        } else if (more >= 16) {
#pragma unroll
            for (int i = 0; i < SU; ++i) sc[i] = v4u{0, 0, 0, 0};
        } else if (blocks >= 16) {
#pragma unroll
            for (int i = 0; i < SU; ++i) {
                v4u t = *(const v4u_byte AQ_GLOBAL*)(scale_row[i] + blocks - 16);
                if (more & 8) t = v4u{t[2], t[3], 0, 0};
                if (more & 4) t = v4u{t[1], t[2], t[3], 0};
                const uint32_t bits = 8 * (more & 3);
                sc[i] = v4u{__builtin_amdgcn_alignbit(t[1], t[0], bits), __builtin_amdgcn_alignbit(t[2], t[1], bits),
                            __builtin_amdgcn_alignbit(t[3], t[2], bits), t[3] >> bits};
            }
        } else {
#pragma unroll
            for (int i = 0; i < SU; ++i) {
                const uint8_t* const row = scale_row[i];
                const int o8 = blocks & 8, o4 = blocks & 12, o2 = blocks & 14;
                const v2u a = o8 ? *(const v2u_byte AQ_GLOBAL*)row : v2u{0, 0};
                const uint32_t b = blocks & 4 ? *(const u32_byte AQ_GLOBAL*)(row + o8) : 0;
                const uint32_t c2 = blocks & 2 ? *(const u16_byte AQ_GLOBAL*)(row + o4) : 0;
                const uint32_t c1 = blocks & 1 ? *(const uint8_t AQ_GLOBAL*)(row + o2) : 0;
                const uint32_t c = blocks & 2 ? c2 | c1 << 16 : c1;
                sc[i] = v4u{o8 ? a[0] : blocks & 4 ? b : c, o8 ? a[1] : blocks & 4 ? c : 0, o8 ? blocks & 4 ? b : c : 0, o4 == 12 ? c : 0};
            }
        }
    };
    uint32_t* const lds_scales = (uint32_t*)(lds + 2 * kBuf);  // [8 words][R]: two words to a chunk
    auto put_scales = [&](int chunk) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < SU; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (NT * SU == R || tid < R) lds_scales[((2 * chunk + k) & 7) * R + tid + NT * i] = sc[i][k];
    };
    v16f32 acc[TN][TM];
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
    // operands of a turn and of the next; a lane's blocks of a chunk are 2 turn + g
    v4u cx[2][TM], cw[2][TN];
    uint32_t sx[2][TM], sw[2][TN];  // scales of a chunk's two halves
    const int place = ((g ^ ((lane >> 1) & 7)) << 4) + r * 128;
    auto read = [&](auto turn, const uint8_t* from) __attribute__((always_inline)) {
        constexpr int Q = decltype(turn)::value;
        const uint8_t* const at = from + (place ^ (32 * Q));
#pragma unroll
        for (int j = 0; j < TM; ++j) cx[Q & 1][j] = *(const v4u*)(at + (wm + 32 * j) * 128);
#pragma unroll
        for (int i = 0; i < TN; ++i) cw[Q & 1][i] = *(const v4u*)(at + (wn + 32 * i) * 128);
    };
    auto read_scales = [&](auto half, int chunk) __attribute__((always_inline)) {
        constexpr int H = decltype(half)::value;
        const uint32_t* const at = lds_scales + ((2 * chunk + H) & 7) * R + r;
#pragma unroll
        for (int j = 0; j < TM; ++j) sx[H][j] = at[wm + 32 * j];
#pragma unroll
        for (int i = 0; i < TN; ++i) sw[H][i] = at[wn + 32 * i];
    };
    auto own_scales = [&](auto half) __attribute__((always_inline)) {  // this lane's blocks to bytes 0 and 2
        constexpr int H = decltype(half)::value;
#pragma unroll
        for (int j = 0; j < TM; ++j) sx[H][j] >>= 8 * g;
#pragma unroll
        for (int i = 0; i < TN; ++i) sw[H][i] >>= 8 * g;
    };
    auto products = [&](auto turn) __attribute__((always_inline)) {
        constexpr int Q = decltype(turn)::value;
        __builtin_amdgcn_sched_barrier(0);  // (the order stays: operands are requested a turn ahead)
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
            for (int j = 0; j < TM; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(cw[Q & 1][i]), operand(cx[Q & 1][j]), acc[i][j], kFp4, kFp4,
                                                                        2 * (Q & 1), (int)sw[Q / 2][i], 2 * (Q & 1), (int)sx[Q / 2][j]);
        __builtin_amdgcn_sched_barrier(0);
    };
    constexpr std::integral_constant<int, 0> q0{};
    constexpr std::integral_constant<int, 1> q1{};
    constexpr std::integral_constant<int, 2> q2{};
    constexpr std::integral_constant<int, 3> q3{};
    fetch_scales(0);
    fetch(0);
    put_scales(0);
    wait_loads<0>();
    lds_barrier();
    fetch(1);
    read(q0, lds);
    read_scales(q0, 0);
    for (int c = 0; c < chunks; ++c) {
        const uint8_t* const now = lds + (c & 1) * kBuf;
        own_scales(q0);
        if ((c & 1) == 0) fetch_scales(8 * c + 16);
        read_scales(q1, c);
        read(q1, now);
        products(q0);
        read(q2, now);
        products(q1);
        own_scales(q1);
        if ((c & 1) == 1) put_scales(c + 1);
        read(q3, now);
        products(q2);
        wait_loads<0>();  // the next chunk is there,
        lds_barrier();    // and all of this one in registers
        fetch(c + 2);
        read(q0, lds + ((c + 1) & 1) * kBuf);
        read_scales(q0, c + 1);
        products(q3);
    }
    wait_loads<0>();  // (chunks behind the last one, which arrive as zeros)
    lds_barrier();
    v4f32 b[TN][4];
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int64_t f = n0 + wn - S + 32 * i + 8 * q + 4 * g + e;
                b[i][q][e] = bias && f < n ? bias[f] : 0.0f;
            }
    const int64_t f0 = n0 + wn - S;
#pragma unroll
    for (int j = 0; j < TM; ++j) {
        const int64_t row = m0 + wm + 32 * j;
        store_rows<T, TN>(lds + wave * (32 * kOutRow<T, TN>), lane, y + row * ldy + f0, ldy, rows - row, n - f0,
                          [&](int i, int q, int e) { return acc[i][j][4 * q + e] + b[i][q][e]; });
    }
}

Blocks blocks_of(const aq_mx4& q) { return {(const uint8_t*)q.d_codes, q.d_scales, blocks32(q.cols)}; }

// Whether the few-row kernel takes a product, by its 16 x 16 tiles, as many workgroups, and the bytes of a row of x, which each of them
// reads and, where they are values, quantizes again; up to a workgroup to a CU always.  us on it / on the tiles, for values with the
// quantization that goes before them.
// Values: 256 tiles  2048 x 2048 bfloat16 4.2 / 9.1, 4096 x 4096 fp32 6.1 / 13.2
//         512        2048 x 2048 bfloat16 5.7 / 9.1, 4096 x 4096 fp32 10.1 / 13.2, 1024 x 8192 18.4 / 21.8
//         1024       512 x 3136 bfloat16 9.7 / 13.1, fp32 15.0 / 13.2;  2048 x 2048 bfloat16 8.5 / 9.2, fp32 10.2 / 9.5
//         1536       1024 x 1024 bfloat16 7.0 / 7.4, fp32 8.4 / 7.6
//         2048       256 x 256 fp32 5.5 / 6.9;  1024 x 512 fp32 6.5 / 6.6 (bfloat16, half as many again, 7.6 / 6.5)
// Blocks: 512 tiles  2048 x 2048 5.7 / 5.8, 512 x 3136 5.8 / 7.8, 1024 x 8192 16.4 / 13.7;  1024  1024 x 512 3.8 / 4.0, 2048 x 2048 9.4 / 5.8
//         2048       256 x 256 4.1 / 4.2, 1024 x 512 5.4 / 4.0
bool few_rows(int64_t rows, int64_t n, int64_t row_bytes, bool values) {
    const int64_t tiles = ((rows + 15) / 16) * ((n + 15) / 16);
    if (values) return tiles <= 512 || row_bytes + 3000 <= 9500000 / tiles;
    return tiles <= 256 || row_bytes + 400 <= 1050000 / tiles;
}

int64_t tiles_of(int64_t rows, int64_t n, int64_t side) { return ((rows + side - 1) / side) * ((n + side - 1) / side); }
// The largest tiles that give every CU one; 0 where no launch holds them.  us on tiles of 64 / 128 / 256: 2048 x 2048, 2048 rows
// 13.3 / 11.7 / 19.0, 8192 rows 42.9 / 31.4 / 25.5; 4096 x 4096, 1024 rows 22.1 / 17.3 / 30.7; 1024 x 1024, 2048 rows 6.2 / 8.0 / 12.3.
int tile_side(int64_t rows, int64_t n) {
    if (tiles_of(rows, n, 256) >= 256) return grid_ok(tiles_of(rows, n, 256), tile_threads(256)) ? 256 : 0;
    return tiles_of(rows, n, 128) >= 256 ? 128 : 64;
}

template <class X, class T>
aq_status launch_rows(const X& x, int64_t rows, const aq_mx4& w, const float* bias, const aq_matrix& y, hipStream_t st) {
    const dim3 grid((unsigned)((w.rows + 15) / 16), (unsigned)((rows + 15) / 16));
    k_mx4_rows<X, T><<<grid, 512, 0, st>>>(x, blocks_of(w), bias, (T*)y.d, y.ld, (int)rows, (int)w.rows, (int)blocks32(w.cols));
    return hip_failed(hipGetLastError()) ? AQ_EHIP : AQ_OK;
}

template <class T, int S>
aq_status launch_tiles(const aq_mx4& x, const aq_mx4& w, const float* bias, const aq_matrix& y, hipStream_t st) {
    constexpr int kLds = 2 * 2 * S * 128 + 8 * 2 * S * 4;
    constexpr int NT = tile_threads(S);
    auto* const k = k_mx4_tiles<T, S, NT>;
    if (!allow_lds<Blocks, T, std::integral_constant<int, S>>((const void*)k, kLds)) return AQ_EHIP;
    k<<<(unsigned)tiles_of(x.rows, w.rows, S), NT, kLds, st>>>(blocks_of(x), blocks_of(w), bias, (T*)y.d, y.ld, (int)x.rows, (int)w.rows,
                                                               (int)blocks32(w.cols));
    return hip_failed(hipGetLastError()) ? AQ_EHIP : AQ_OK;
}

}  // namespace

int64_t mx4_linear_workspace(int64_t rows, int64_t n, int64_t k) {
    if (few_rows(rows, n, 4 * k, true)) return 0;  // (whatever the type)
    const int64_t b = rows * blocks32(k);
    return 16 * b + (b + 15) / 16 * 16;
}

aq_status launch_mx4_matmul(const aq_mx4& x, const aq_mx4& w, const float* bias, const aq_matrix& y, hipStream_t st) {
    return with_dtype(y.dtype, [&](auto t) {
        using T = decltype(t);
        if (few_rows(x.rows, w.rows, 16 * blocks32(x.cols), false)) return launch_rows<Blocks, T>(blocks_of(x), x.rows, w, bias, y, st);
        switch (tile_side(x.rows, w.rows)) {
            case 256: return launch_tiles<T, 256>(x, w, bias, y, st);
            case 128: return launch_tiles<T, 128>(x, w, bias, y, st);
            case 64: return launch_tiles<T, 64>(x, w, bias, y, st);
        }
        return AQ_ESHAPE;
    });
}

aq_status launch_mx4_linear(const aq_matrix& x, const aq_mx4& w, const float* bias, const aq_matrix& y, void* ws, hipStream_t st) {
    if (few_rows(x.rows, w.rows, x.cols * (int64_t)dtype_bytes(x.dtype), true))
        return with_dtype(x.dtype, [&](auto t) {
            using T = decltype(t);
            return launch_rows<Values<T>, T>(Values<T>{(const T*)x.d, x.ld, (int)x.cols}, x.rows, w, bias, y, st);
        });
    if (!tile_side(x.rows, w.rows)) return AQ_ESHAPE;  // (before the quantization)
    const int64_t b = x.rows * blocks32(x.cols);
    const aq_mx4 q = {ws, (uint8_t*)ws + 16 * b, x.rows, x.cols};
    const aq_status s = launch_mx4_quantize(x, q, st);
    return s != AQ_OK ? s : launch_mx4_matmul(q, w, bias, y, st);
}

}  // namespace aq
