// The gradients of a fully connected layer from what it keeps in few bits:
//   weight gradient  dw[n][k] = sum_row dy[row][n] x8[row][k]      x8: the 8-bit checkpoint of its input
//   input gradient   dx[row][k] = sum_n dy[row][n] w4[n][k]        w4: its microscaled 4-bit weights
// Both are C[m][c] = sum_t A[m][t] B[t][c] on the bf16 matrix cores, without a rounding in front of the sums: a code of
// either format times its power of two has at most seven significant bits, so it is a bf16 value (4-bit values of 2^128 and more are
// infinities), and a value of dy is the sum of one (bfloat16), two (binary16) or three (fp32) bf16 values.
//
// Bound by the matrix cores' power and by what feeds them: 65536 x 2048 x 2048 in bfloat16 takes 521 to 555 us back to back
// (1.02 PFLOP/s; 471 alone), the input gradient 8192 x 2048 x 2048 61 us (1.13 PFLOP/s), where a loop of nothing but these
// products on such values reaches 1.88 PFLOP/s at the clock that is left and a large library product 1.21.  binary16 takes twice
// and fp32 three times the products (610 and 410 TFLOP/s).
//
// A workgroup's 32 t of both operands go through LDS.  B lies there as it does in memory, t by t (and so does A for the weight
// gradient), and is transposed on its way to the registers: ds_read_b64_tr_b16 hands lane i of 16 the four t of column i out of
// four rows of 16 columns.
#include <utility>

#include "learner.hpp"
#include "product_device.hpp"

namespace aq {
namespace {

typedef short v4s16 __attribute__((ext_vector_type(4)));

constexpr int grad_buffers(int bytes) { return 3 * bytes <= kMostLds ? 3 : 2; }

template <class T>
constexpr int kParts = std::is_same<T, float>::value ? 3 : std::is_same<T, f16_t>::value ? 2 : 1;

// Eight values as P bf16 parts, each the rest of the one before cut to bf16 (cut, not rounded: no part overflows, and three times
// eight bits are fp32's 24).  An infinity's or a NaN's first part is one itself (a NaN is made quiet, so that the cut leaves it one);
// the others are those of the largest number, of an infinity's sign: no product of theirs overflows to the other infinity.
template <class T, int P>
__device__ __forceinline__ void split(const Piece<T>& in, v4u (&out)[P]) {
    if constexpr (P == 1) {
        out[0] = v4u{in.w[0], in.w[1], in.w[2], in.w[3]};
    } else {
        float v[8];
        in.get(v);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = __builtin_canonicalizef(v[j]);
#pragma unroll
        for (int q = 0; q < P; ++q) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                out[q][j] = __builtin_amdgcn_perm(__float_as_uint(v[2 * j + 1]), __float_as_uint(v[2 * j]), 0x07060302u);
            if (q + 1 < P) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (q == 0) v[j] = __builtin_amdgcn_fmed3f(v[j], -3.40282347e38f, 3.40282347e38f);
                    v[j] -= __uint_as_float(__float_as_uint(v[j]) & 0xffff0000u);
                }
            }
        }
    }
}

// ---- LDS tiles of 32 t
// [t][S columns]: 32-byte pieces of a row, piece p of row t in place p ^ 2 (t mod 4), so that the four rows and two pieces which 32 lanes
// of a transposing read take lie in different banks
template <int S>
__device__ __forceinline__ int t_at(int t, int col) {  // byte address of column col (a multiple of 8) of row t
    return t * 2 * S + (((col >> 4) ^ ((t & 3) << 1 & (S / 16 - 1))) << 5) + ((col & 8) << 1);
}
// 32 columns from col on, 16 t from t0 on, as an MFMA operand: lane l has column l mod 32, t = 8 (l / 32) .. + 7
template <int S>
__device__ __forceinline__ v8bf16 t_operand(const uint8_t* tile, int t0, int col, int lane) {
    typedef __attribute__((address_space(3))) v4s16* lds_ptr;
    const int i = lane & 15, t = t0 + 8 * (lane >> 5) + (i >> 2);
    const uint8_t* p = tile + t_at<S>(t, col + (lane & 16)) + (i & 3) * 8;
    const v4s16 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)p);
    const v4s16 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p + 4 * 2 * S));
    return __builtin_bit_cast(v8bf16, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}
// [row m][32 t]: 16-byte pieces, piece p of row m in place p ^ (m / 4 mod 4)
__device__ __forceinline__ int m_at(int m, int piece) { return m * 64 + ((piece ^ ((m >> 2) & 3)) << 4); }

// ---- the operands.  Of 32 t and S columns (or rows) each thread fetches kUnits units of eight values into registers and later puts them
// into LDS as bf16.  Loads go through windows on the matrix (see Window).  Columns of an operand that do not exist only reach results
// that are not stored.
// A matrix in whole words of memory: from the word of its first element to that of its last.
struct Words {
    const uint8_t* base;
    int64_t size;
    int skew;  // bytes in front of the first element
    int64_t ld, rows;
};
template <class T>
Words words_of(const aq_matrix& m) {
    const uintptr_t first = (uintptr_t)m.d, end = first + (m.rows ? ((m.rows - 1) * m.ld + m.cols) * sizeof(T) : 0);
    const uintptr_t base = first & ~(uintptr_t)3;
    return {(const uint8_t*)base, (int64_t)(((end + 3) & ~(uintptr_t)3) - base), (int)(first - base), m.ld, m.rows};
}
// Eight values `at` bytes from a window's beginning.  ODD: 16-bit values of which some pieces begin in the middle of a word; they are
// shifted into place out of five words, so that no load leaves the matrix's words.
template <class T, bool ODD>
__device__ __forceinline__ void load_piece(Piece<T>& q, const Window& w, int at) {
    if constexpr (ODD) {
        const v4u v = __builtin_amdgcn_raw_buffer_load_b128(w.r, at & ~3, 0, 0);
        const uint32_t last = __builtin_amdgcn_raw_buffer_load_b32(w.r, (at & ~3) + 16, 0, 0), by = (at & 2) * 8;
#pragma unroll
        for (int i = 0; i < 4; ++i) q.w[i] = __builtin_amdgcn_alignbit(i < 3 ? v[i < 3 ? i + 1 : 0] : last, v[i], by);
    } else {
#pragma unroll
        for (int i = 0; i < Piece<T>::kWords; i += 4) {
            const v4u v = __builtin_amdgcn_raw_buffer_load_b128(w.r, at, 0, 0);
#pragma unroll
            for (int j = 0; j < 4; ++j) q.w[i + j] = v[j];
            at += 16;
        }
    }
}
template <class T, bool ANY>
constexpr bool kOdd = ANY && sizeof(T) == 2;
// Where a thread's units lie in a window, which move 32 t with every fetch.  After `turns` fetches of all units the window itself moves
// on, so that no offset passes 31 bits.
template <int U>
struct Track {
    Window w;
    const uint8_t* base;
    int64_t at, size;  // the window's beginning, a multiple of 4; what it may show, from base on
    int step;          // bytes
    int off[U];
    __device__ __forceinline__ void begin(const uint8_t* b, int64_t first, int64_t bytes, int per_step) {
        base = b;
        at = first;
        size = bytes;
        step = per_step;
        w.set(base, at, size);
    }
    __device__ __forceinline__ void move(int turns) {
        at += (int64_t)turns * step;
        w.set(base, at, size);
#pragma unroll
        for (int i = 0; i < U; ++i) off[i] -= turns * step;
    }
};
// most turns for which offsets stay within 31 bits, some fetches ahead included
inline int track_turns(int64_t step) { return (int)(0x7fffffff / step - 5); }

// a thread's place among those that share a tile of S x S (only the smallest tiles are shared by several groups)
template <int S>
__device__ __forceinline__ uint32_t thread_of() {
    return S == 64 ? threadIdx.x % tile_threads(S) : threadIdx.x;
}

// dy with t along the rows (weight gradient): [t][m].  ANY: rows of any alignment.
template <class T, int S, bool ANY>
struct DyRows {
    static constexpr int P = kParts<T>, NT = tile_threads(S), kUnits = 4 * S / NT, kPlane = 32 * 2 * S, kPer = S / 8;
    static constexpr int kSets = P == 1 || S < 256 ? 2 : 1;
    static constexpr bool kSums = true;
    Words d;
    Track<kUnits> k;
    int left;
    Piece<T> in[kSets][kUnits];
    __device__ __forceinline__ void begin(int64_t m0, int64_t t0, int64_t t_end) {
        const int64_t byte = (t0 * d.ld + m0) * (int64_t)sizeof(T) + d.skew;
        const int64_t most = (t_end * d.ld * (int64_t)sizeof(T) + d.skew + 3) & ~(int64_t)3;  // (no row behind the slice's)
        k.begin(d.base, byte & ~(int64_t)3, d.size < most ? d.size : most, 32 * (int)d.ld * (int)sizeof(T));
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
            const int u = thread_of<S>() + NT * i;
            k.off[i] = ((int)byte & 3) + ((u / kPer) * (int)d.ld + 8 * (u % kPer)) * (int)sizeof(T);
        }
        left = (int)(t_end - t0) - thread_of<S>() / kPer;
    }
    __device__ __forceinline__ void move(int turns) { k.move(turns); }
    __device__ __forceinline__ void fetch(int set, int i) {
        int at = k.off[i];
        k.off[i] += k.step;
        if constexpr (kOdd<T, ANY>) {  // (the last word may hold what would be the first value of a row behind the last)
            if (left <= NT / kPer * i) at = Window::kOutside;
            if (i == kUnits - 1) left -= 32;
        }
        load_piece<T, kOdd<T, ANY>>(in[set][i], k.w, at);
    }
    __device__ __forceinline__ void put(int set, int i, uint8_t* to) const {
        const int u = thread_of<S>() + NT * i;
        v4u q[P];
        split<T, P>(in[set][i], q);
#pragma unroll
        for (int p = 0; p < P; ++p) *(v4u*)(to + p * kPlane + t_at<S>(u / kPer, 8 * (u % kPer))) = q[p];
    }
    static __device__ __forceinline__ v8bf16 operand(const uint8_t* tile, int t0, int m, int lane) { return t_operand<S>(tile, t0, m, lane); }
};
// dy with t along the columns (input gradient): [m][t].  ANY: rows of any alignment, which may end inside a piece whose other
// values are the next row's.
template <class T, int S, bool ANY>
struct DyCols {
    static constexpr int P = kParts<T>, NT = tile_threads(S), kUnits = 4 * S / NT, kPlane = 32 * 2 * S;
    static constexpr int kSets = P == 1 || S < 256 ? 2 : 1;
    static constexpr bool kSums = false;
    Words d;
    Track<kUnits> k;
    int left[kSets], next;  // values that exist of this thread's pieces
    Piece<T> in[kSets][kUnits];
    __device__ __forceinline__ void begin(int64_t m0, int64_t t0, int64_t t_end) {
        const int64_t byte = (m0 * d.ld + t0) * (int64_t)sizeof(T) + d.skew;
        k.begin(d.base, byte & ~(int64_t)3, d.size, 32 * (int)sizeof(T));
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
            const int u = thread_of<S>() + NT * i;
            k.off[i] = ((int)byte & 3) + ((u >> 2) * (int)d.ld + 8 * (u & 3)) * (int)sizeof(T);
        }
        next = (int)(t_end - t0) - 8 * (thread_of<S>() & 3);
    }
    __device__ __forceinline__ void move(int turns) { k.move(turns); }
    __device__ __forceinline__ void fetch(int set, int i) {
        load_piece<T, kOdd<T, ANY>>(in[set][i], k.w, next > 0 ? k.off[i] : Window::kOutside);
        k.off[i] += k.step;
        if (i == kUnits - 1) {
            left[set] = next;
            next -= 32;
        }
    }
    __device__ __forceinline__ void put(int set, int i, uint8_t* to) const {
        const int u = thread_of<S>() + NT * i;
        Piece<T> own = in[set][i];
        if constexpr (ANY) {
            const int n = left[set];
#pragma unroll
            for (int j = 0; j < Piece<T>::kWords; ++j) {
                if constexpr (sizeof(T) == 4) own.w[j] = j < n ? own.w[j] : 0;
                else own.w[j] &= 2 * j + 1 < n ? 0xffffffffu : 2 * j < n ? 0xffffu : 0u;
            }
        }
        v4u q[P];
        split<T, P>(own, q);
#pragma unroll
        for (int p = 0; p < P; ++p) *(v4u*)(to + p * kPlane + m_at(u >> 2, u & 3)) = q[p];
    }
    static __device__ __forceinline__ v8bf16 operand(const uint8_t* tile, int t0, int m, int lane) {
        return *(const v8bf16*)(tile + m_at(m + (lane & 31), t0 / 8 + (lane >> 5)));
    }
};
// rows of a checkpoint (CODE bytes of codes to eight values: 8) or of 4-bit weights (4)
template <int S, int SETS, int CODE>
struct BlockRows {
    static constexpr int NT = tile_threads(S), kUnits = 4 * S / NT, kPlane = 32 * 2 * S, kPer = S / 8;
    typedef typename std::conditional<CODE == 8, v2u, uint32_t>::type Codes;
    const uint8_t* codes;
    const uint8_t* scales;
    int64_t blocks, rows;
    Track<kUnits> kc, ks;
    Codes c[SETS][kUnits];
    uint32_t s[SETS][kUnits];
    __device__ __forceinline__ void begin(int64_t c0, int64_t t0, int64_t t_end) {
        const int64_t last = rows < t_end ? rows : t_end;
        const int skew = (int)((uintptr_t)scales & 3);
        const int64_t byte = t0 * blocks + (c0 >> 5) + skew;
        kc.begin(codes, (t0 * blocks * 4 + c0 / 8) * CODE, last * blocks * 4 * CODE, 32 * (int)blocks * 4 * CODE);
        ks.begin(scales - skew, byte & ~(int64_t)3, last * blocks + skew, 32 * (int)blocks);
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
            const int u = thread_of<S>() + NT * i, t = u / kPer, piece = u % kPer;
            kc.off[i] = (t * (int)blocks * 4 + piece) * CODE;
            ks.off[i] = ((int)byte & 3) + t * (int)blocks + (piece >> 2);
        }
    }
    __device__ __forceinline__ void move(int turns) {
        kc.move(turns);
        ks.move(turns);
    }
    __device__ __forceinline__ void fetch(int set, int i) {
        if constexpr (CODE == 8) c[set][i] = __builtin_bit_cast(v2u, __builtin_amdgcn_raw_buffer_load_b64(kc.w.r, kc.off[i], 0, 0));
        else c[set][i] = __builtin_amdgcn_raw_buffer_load_b32(kc.w.r, kc.off[i], 0, 0);
        s[set][i] = __builtin_amdgcn_raw_buffer_load_b8(ks.w.r, ks.off[i], 0, 0);
        kc.off[i] += kc.step;
        ks.off[i] += ks.step;
    }
    __device__ __forceinline__ void put(int set, int i, uint8_t* to) const {
        const int u = thread_of<S>() + NT * i;
        v4u o;
        if constexpr (CODE == 8) {
            float v[8];
            ckpt8_values(c[set][i], ckpt8_step(s[set][i]), v);
            Piece<bf16_t> q;
            q.set(v);
            o = v4u{q.w[0], q.w[1], q.w[2], q.w[3]};
        } else {
            const float step = mx4_step(s[set][i]);
            const uint32_t w = c[set][i];
            o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, step, 0));
            o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, step, 1));
            o[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, step, 2));
            o[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, step, 3));
        }
        *(v4u*)(to + t_at<S>(u / kPer, 8 * (u % kPer))) = o;
    }
};

// calls f(integral_constant i) for i = 0 .. N - 1
template <int N, class F, int... I>
__device__ __forceinline__ void static_for(F&& f, std::integer_sequence<int, I...>) {
    (f(std::integral_constant<int, I>()), ...);
}
template <int N, class F>
__device__ __forceinline__ void static_for(F&& f) {
    static_for<N>(f, std::make_integer_sequence<int, N>());
}

// C tile of S x S, a wavefront takes S / 2 rows and NC * 32 columns of it.  Slice z takes t in [z * chunks * 32, + chunks * 32) and
// writes its own C (and its own sums of A over t, where `sums` is given).  While the products of one 32 t run, the next 32 t go from
// registers to LDS, unit by unit, and one or two more are on their way from memory behind them (three or four gain nothing); with
// three buffers the barrier lies two groups of products before the end, and the next operands are read behind it.
//
// H: as many groups of wavefronts share a tile, each with buffers of its own and a slice of its own; their sums join in LDS, in their
// order.  Two halve the chain of chunks that bounds small products, without slices' way through memory: input gradient 300 x 403 x
// 1111 binary16 9.7 us with one, 8.5 with two, 8.8 with four.
template <class A, class B, class T, int S, int H>
__global__ void __launch_bounds__(H * tile_threads(S), 1)
    k_grad(A a, B b, T* __restrict__ out, int64_t ld, int64_t out_stride, float* __restrict__ sums, int64_t mn, int64_t cn, int64_t tn,
           int chunks, int turns) {
    constexpr int P = A::P, NT = tile_threads(S), N = S / 64, NC = S / (NT / 128) / 32;
    constexpr int kBuf = P * A::kPlane + B::kPlane, kBufs = grad_buffers(H * kBuf);
    constexpr int G = 2 * P * N;  // groups of NC products: 16 t, part, row tile
    static_assert(NT / 64 * 32 * kOutRow<T, NC> <= kBufs * kBuf, "results leave through the buffers");
    static_assert(H == 1 || NT * (N * NC * 64 + 4) <= kBufs * kBuf, "and so do a group's sums");
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const int group = H > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / NT) : 0;
    const int own = group * (kBufs * kBuf);  // where this group's buffers begin
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(thread_of<S>() >> 6), r = lane & 31, g = lane >> 5;
    const Place at = place_of_workgroup((uint32_t)((mn + S - 1) / S), (uint32_t)((cn + S - 1) / S));
    const int64_t m0 = (int64_t)at.m * S, c0 = (int64_t)at.c * S;
    const int wm = (wave & 1) * (S / 2), wc = (wave >> 1) * (32 * NC);
    const int64_t t_all = (int64_t)at.z * H * chunks * 32, t_first = t_all + (int64_t)group * chunks * 32;
    const int64_t t_behind = tn;
    if (t_first + (int64_t)chunks * 32 < tn) tn = t_first + (int64_t)chunks * 32;
    a.begin(m0, t_first, tn);
    b.begin(c0, t_first, tn);
    v16f32 acc[N][NC];
    float acc_sum = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
#pragma unroll
        for (int j = 0; j < NC; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
    }
    auto fetch_all = [&](int set) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < A::kUnits; ++i) {
            a.fetch(set, i);
            b.fetch(set, i);
        }
    };
    // A wavefront begins with the row tile of its own number among those that share the rows, whose sums it takes: all rows' sums at a
    // fraction of the cost that one wavefront's would have, and no jumps.
    auto tile_of = [&](int i) __attribute__((always_inline)) { return A::kSums ? (i + (wave >> 1)) % N : i; };
    // group q: 16 t from 16 (q / (P N)), part P - 1 - q / N mod P (the smallest first), row tile q mod N
    auto read_a = [&](const uint8_t* tile, int q) __attribute__((always_inline)) {
        return A::operand(tile + (P - 1 - q / N % P) * A::kPlane, 16 * (q / (P * N)), wm + 32 * tile_of(q % N), lane);
    };
    auto read_b = [&](const uint8_t* tile, int j) __attribute__((always_inline)) {  // j: 16 t from 16 (j / NC), column tile j mod NC
        return t_operand<S>(tile + P * A::kPlane, 16 * (j / NC), wc + 32 * (j % NC), lane);
    };
    {
        const v2bf16 ones = __builtin_bit_cast(v2bf16, 0x3f803f80u);
#pragma unroll
        for (int i = 0; i < A::kSets; ++i) fetch_all(i);
#pragma unroll
        for (int i = 0; i < A::kUnits; ++i) {
            a.put(0, i, lds + own);
            b.put(0, i, lds + own + P * A::kPlane);
        }
        fetch_all(0);
        lds_barrier();
        v8bf16 ob[2 * NC], oa;
#pragma unroll
        for (int j = 0; j < 2 * NC; ++j) ob[j] = read_b(lds + own, j);
        oa = read_a(lds + own, 0);
        int now = own;
        auto step = [&](auto then) __attribute__((always_inline)) {
            constexpr int kThen = decltype(then)::value;  // the set that holds the next 32 t
            const uint8_t* const tile = lds + now;
            now = now + kBuf == own + kBufs * kBuf ? own : now + kBuf;
            uint8_t* const next = lds + now;
            v8bf16 ob_next[2 * NC], oa_next;
            constexpr int kTasks = 2 * A::kUnits, kSlots = G > 2 ? G - 2 : 1;
            static_for<G>([&](auto group) __attribute__((always_inline)) {
                constexpr int q = decltype(group)::value;
                if (kBufs == 3 && q >= kSlots) {
                    if (q == kSlots) lds_barrier();
#pragma unroll
                    for (int j = (q - kSlots) * 2 * NC / (G - kSlots); j < (q - kSlots + 1) * 2 * NC / (G - kSlots); ++j)
                        ob_next[j] = read_b(next, j);
                }
                if (q + 1 < G) oa_next = read_a(tile, q + 1);
                else if (kBufs == 3) oa_next = read_a(next, 0);
#pragma unroll
                for (int j = 0; j < NC; ++j)
                    acc[q % N][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ob[q / (P * N) * NC + j], oa, acc[q % N][j], 0, 0, 0);
                if constexpr (A::kSums && q % N == 0) {
                    const v4u w = __builtin_bit_cast(v4u, oa);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t pair = w[j];  // (a vector's element itself is not cast right: the first one is taken for all)
                        acc_sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(v2bf16, pair), ones, acc_sum, false);
                    }
                }
#pragma unroll
                for (int k = 0; k < kTasks; ++k)
                    if (k * kSlots / kTasks == q) {
                        if (k & 1) {
                            b.put(kThen, k / 2, next + P * A::kPlane);
                            b.fetch(kThen, k / 2);
                        } else {
                            a.put(kThen, k / 2, next);
                            a.fetch(kThen, k / 2);
                        }
                    }
                oa = oa_next;
                __builtin_amdgcn_sched_barrier(0);  // (loads stay in the order in which they are waited for)
            });
            if constexpr (kBufs == 3) {
#pragma unroll
                for (int j = 0; j < 2 * NC; ++j) ob[j] = ob_next[j];
            } else {
                lds_barrier();
#pragma unroll
                for (int j = 0; j < 2 * NC; ++j) ob[j] = read_b(next, j);
                oa = read_a(next, 0);
            }
        };
        int to_move = turns;
        int left = (int)(tn - t_first);
        if (H > 1)  // the first group's, which has the most
            left = (int)(t_behind - t_all < (int64_t)chunks * 32 ? t_behind - t_all : (int64_t)chunks * 32);
        for (; left > 0; left -= 64) {  // (32 t behind the end are zeros)
            step(std::integral_constant<int, A::kSets - 1>());
            step(std::integral_constant<int, 0>());
            if ((to_move -= 2) <= 0) {
                a.move(turns);
                b.move(turns);
                to_move = turns;
            }
        }
    }
    out += at.z * out_stride;
    wait_loads<0>();
    lds_barrier();  // (every wavefront has read its last operands)
    if constexpr (H > 1) {
        constexpr int kEach = N * NC * 4;  // v4f32 of a thread
        const int thread = thread_of<S>();
        if (group) {
#pragma unroll
            for (int k = 0; k < kEach; ++k) {
                const v16f32& v = acc[k / (NC * 4)][k / 4 % NC];
                ((v4f32*)(lds + own))[k * NT + thread] = v4f32{v[k % 4 * 4], v[k % 4 * 4 + 1], v[k % 4 * 4 + 2], v[k % 4 * 4 + 3]};
            }
            ((float*)(lds + own))[kEach * 4 * NT + thread] = acc_sum;
        }
        lds_barrier();
        if (group) return;
        for (int h = 1; h < H; ++h) {
            const uint8_t* const from = lds + h * (kBufs * kBuf);
#pragma unroll
            for (int k = 0; k < kEach; ++k) {
                const v4f32 v = ((const v4f32*)from)[k * NT + thread];
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[k / (NC * 4)][k / 4 % NC][k % 4 * 4 + e] += v[e];
            }
            acc_sum += ((const float*)from)[kEach * 4 * NT + thread];
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int64_t row = m0 + wm + 32 * tile_of(i), m = row + r;
        store_rows<T, NC>(lds + wave * (32 * kOutRow<T, NC>), lane, out + row * ld + c0 + wc, ld, mn - row, cn - c0 - wc,
                          [&](int j, int q, int e) { return acc[i][j][4 * q + e]; });
        if constexpr (A::kSums) {
            if (i == 0) {
                const float s = acc_sum + __shfl_xor(acc_sum, 32, 64);
                if (sums && at.c == 0 && wave >> 1 < N && g == 0 && m < mn) sums[at.z * mn + m] = s;
            }
        }
    }
}

constexpr int kJoinThreads = 256;
constexpr int64_t kMostThreads = 0xffffffffLL;  // of a launch

// the slices' results join, in their order, and are rounded; dy's sums behind them
template <class T>
__global__ void __launch_bounds__(kJoinThreads) k_grad_join(const float* __restrict__ part, int slices, int64_t m, int64_t c, T* __restrict__ out,
                                                   int64_t ld, const float* __restrict__ part_sums, float* __restrict__ sums) {
    const int64_t i = (int64_t)blockIdx.x * kJoinThreads + threadIdx.x;
    auto total = [slices](const float* p, int64_t step) __attribute__((always_inline)) {
        float s = 0.0f;
        int k = 0;
        for (; k + 8 <= slices; k += 8) {  // eight on their way at a time
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = p[(k + j) * step];
#pragma unroll
            for (int j = 0; j < 8; ++j) s += v[j];
        }
        for (; k < slices; ++k) s += p[k * step];
        return s;
    };
    if (i < m * c) out[i / c * ld + i % c] = (T)total(part + i, m * c);
    else if (sums && i < m * c + m) sums[i - m * c] = total(part_sums + (i - m * c), m);
}

// how a product of m x c over t runs: tiles of s x s, z times h slices of `chunks` (an even number) times 32 t, h of them in one workgroup
struct Plan {
    int s, z, h, chunks;
};
// The tile and the slices by an estimate in us: what a launch takes besides its chunks; the chunks of a workgroup one after the
// other, each as long as `alone` while few workgroups are about and `full` while as many as fit are (`at_once`); the join's launch
// and bytes.  Fitted to weight gradients of 2048 rows with every tile in one slice, us on tiles of 64 / 128 / 256:
//   bfloat16 2048 x 2048  51.1 / 38.4 / 54.8,   1024 x 1024 20.5 / 32.9 / 50.4,   128 x 128 18.5 / 31.3 / 49.1 (256 rows 4.9 / 7.7 / 12.1)
//   binary16              73.2 / 55.8 / 97.1,               30.9 / 47.2 / 93.8,             27.8 / 46.2 / 91.9 (6.2 / 9.8 / 17.6)
//   fp32                 103.4 / 76.1 / 137.5,              37.9 / 63.9 / 135.8,            33.7 / 61.7 / 132.5 (6.9 / 11.9 / 23.1)
// and with two groups to a tile of 64
//   bfloat16              50.3, 16.4, 13.7 (4.9),   binary16 75.3, 24.3, 21.0 (5.8),   fp32 115.8, 29.9, 25.4 (6.4)
// (the fitted figures of two groups are a little below these, as other shapes gave them on the same machine as the others).
constexpr int kGroups = 2;  // of wavefronts, where a workgroup has several
struct Kind {
    int s, h;
    struct {
        int bits;  // 2^bits workgroups at once
        float launch, alone, full;
    } cost[3];  // of bfloat16, binary16, fp32
};
struct Plans {
    Plan of[3];
    int most_slices;  // the scratch's, which is the same for every type
};
Plans plans(int64_t m, int64_t c, int64_t t) {
    constexpr Kind kinds[] = {{64, 1, {{10, 3.1f, 0.23f, 0.75f}, {10, 3.1f, 0.40f, 1.10f}, {10, 3.1f, 0.48f, 1.57f}}},
                              {64, kGroups, {{9, 3.6f, 0.29f, 0.66f}, {9, 3.6f, 0.50f, 1.00f}, {8, 3.7f, 0.62f, 0.76f}}},
                              {128, 1, {{9, 4.3f, 0.42f, 0.86f}, {9, 4.6f, 0.65f, 1.52f}, {8, 4.8f, 0.89f, 1.20f}}},
                              {256, 1, {{8, 6.8f, 0.66f, 1.07f}, {8, 7.0f, 1.33f, 1.75f}, {8, 7.4f, 1.95f, 2.60f}}}};
    const int32_t all = (int32_t)((t + 31) / 32);
    const Plan none{64, 1, 1, (all + 1) & ~1};
    Plans best{{none, none, none}, 1};
    float least[3] = {3.0e38f, 3.0e38f, 3.0e38f};
    for (const Kind& k : kinds) {
        const int64_t tiles = ((m < 1 ? 1 : m) + k.s - 1) / k.s * ((c + k.s - 1) / k.s), threads = k.h * tile_threads(k.s);
        for (int32_t want = k.h; want <= 64 && (want == 1 || 2 * want <= all); want *= 2) {
            const int32_t chunks = ((all + want - 1) / want + 1) & ~1, z = chunks ? (all + chunks * k.h - 1) / (chunks * k.h) : 1;
            // (256 CUs; the last turn is as long as a whole one)
            const int64_t wgs = tiles * z, busy = wgs <= 256 ? wgs : (wgs + 255) / 256 * 256;
            if (wgs * threads > kMostThreads || (z > 1 && m * c + m > kMostThreads - kJoinThreads)) continue;  // (no launch holds them)
            const float join = z > 1 ? 2.3f + 0.02f * (float)z + (float)(z * m * c * 4) * (1.0f / 3.5e6f) : 0.0f;
            for (int i = 0; i < 3; ++i) {
                const auto& cost = k.cost[i];
                const int64_t turns = (busy + (1 << cost.bits) - 1) >> cost.bits;
                const float full = (float)busy * (1.0f / (float)(1 << cost.bits));
                const float chunk = turns > 1 ? cost.full * (float)turns : cost.alone + (cost.full - cost.alone) * full * full;
                const float us = cost.launch + join + (float)chunks * chunk;
                if (us < least[i]) {
                    least[i] = us;
                    best.of[i] = {k.s, z, k.h, chunks};
                }
            }
        }
    }
    for (const Plan& p : best.of) best.most_slices = p.z > best.most_slices ? p.z : best.most_slices;
    return best;
}
int type_of(int32_t dtype) { return dtype == AQ_BF16 ? 0 : dtype == AQ_F16 ? 1 : 2; }
int64_t slices_bytes(int64_t z, int64_t values) { return z > 1 ? z * values * (int64_t)sizeof(float) : 0; }

template <class A, class B, class T, int S, int H>
aq_status launch_groups(const A& a, const B& b, T* out, int64_t ld, int64_t stride, float* sums, int64_t m, int64_t c, int64_t t,
                        const Plan& p, int64_t bytes_per_t, hipStream_t st) {
    constexpr int kBuf = A::P * A::kPlane + B::kPlane, kLds = H * grad_buffers(H * kBuf) * kBuf;
    static_assert(kLds <= kMostLds, "");
    const int64_t x = (m + S - 1) / S, y = (c + S - 1) / S;
    if (!grid_ok(x * y * p.z, H * tile_threads(S))) return AQ_ESHAPE;
    auto* const k = k_grad<A, B, T, S, H>;
    if (!allow_lds<A, B, T, std::integral_constant<int, S>, std::integral_constant<int, H>>((const void*)k, kLds)) return AQ_EHIP;
    k<<<(unsigned)(x * y * p.z), H * tile_threads(S), kLds, st>>>(a, b, out, ld, stride, sums, m, c, t, p.chunks,
                                                               track_turns(32 * bytes_per_t) & ~1);
    return hip_failed(hipGetLastError()) ? AQ_EHIP : AQ_OK;
}
template <class A, class B, class T, int S>
aq_status launch(const A& a, const B& b, T* out, int64_t ld, int64_t stride, float* sums, int64_t m, int64_t c, int64_t t, const Plan& p,
                 int64_t bytes_per_t, hipStream_t st) {
    if constexpr (S == 64) {
        if (p.h > 1) return launch_groups<A, B, T, S, kGroups>(a, b, out, ld, stride, sums, m, c, t, p, bytes_per_t, st);
    }
    return launch_groups<A, B, T, S, 1>(a, b, out, ld, stride, sums, m, c, t, p, bytes_per_t, st);
}
template <class T>
aq_status join(const float* part, const Plan& p, int64_t m, int64_t c, T* out, int64_t ld, const float* part_sums, float* sums,
               hipStream_t st) {
    k_grad_join<T><<<(unsigned)((m * c + m + kJoinThreads - 1) / kJoinThreads), kJoinThreads, 0, st>>>(part, p.z, m, c, out, ld, part_sums, sums);
    return hip_failed(hipGetLastError()) ? AQ_EHIP : AQ_OK;
}
template <class Go>
aq_status with_tile(int s, Go&& go) {
    if (s == 256) return go(std::integral_constant<int, 256>());
    if (s == 128) return go(std::integral_constant<int, 128>());
    return go(std::integral_constant<int, 64>());
}
// whether a matrix's pieces of eight values begin at whole words and, with `whole`, end with its rows
template <class T>
bool any_pieces(const aq_matrix& m, bool whole) {
    return (sizeof(T) == 2 && ((uintptr_t)m.d & 3 || m.ld & 1)) || (whole && m.cols % 8);
}

}  // namespace

int64_t weight_grad_workspace(int64_t rows, int64_t n, int64_t k) { return slices_bytes(plans(n, k, rows).most_slices, n * k + n); }

aq_status launch_weight_grad(const aq_matrix& dy, const aq_ckpt8& kept, const aq_matrix& dw, float* db, void* ws, uint64_t ws_bytes,
                             hipStream_t st) {
    const int64_t n = dy.cols, k = kept.cols, rows = dy.rows;
    const Plans all = plans(n, k, rows);
    const Plan p = all.of[type_of(dy.dtype)];
    const bool split_t = p.z > 1;
    if (!workspace_ok(ws, ws_bytes, slices_bytes(all.most_slices, n * k + n))) return AQ_EINVAL;
    float* const out = split_t ? (float*)ws : (float*)dw.d;
    float* const sums = !db ? nullptr : split_t ? (float*)ws + p.z * n * k : db;
    const aq_status s = with_dtype(dy.dtype, [&](auto t) {
        using T = decltype(t);
        return with_tile(p.s, [&](auto sc) {
            constexpr int S = decltype(sc)::value, kSets = DyRows<T, S, false>::kSets;
            const int64_t code_bytes = 32 * blocks32(k), dy_bytes = dy.ld * (int64_t)sizeof(T);
            const int64_t bytes_per_t = dy_bytes > code_bytes ? dy_bytes : code_bytes, ld = split_t ? k : dw.ld;
            const BlockRows<S, kSets, 8> b{(const uint8_t*)kept.d_codes, kept.d_scales, blocks32(k), rows};
            if constexpr (sizeof(T) == 2) {
                if (any_pieces<T>(dy, false))
                    return launch<DyRows<T, S, true>, BlockRows<S, kSets, 8>, float, S>({words_of<T>(dy)}, b, out, ld, n * k, sums, n, k, rows, p,
                                                                                       bytes_per_t, st);
            }
            return launch<DyRows<T, S, false>, BlockRows<S, kSets, 8>, float, S>({words_of<T>(dy)}, b, out, ld, n * k, sums, n, k, rows, p,
                                                                               bytes_per_t, st);
        });
    });
    if (s != AQ_OK || !split_t) return s;
    return join((const float*)ws, p, n, k, (float*)dw.d, dw.ld, sums, db, st);
}

int64_t input_grad_workspace(int64_t rows, int64_t n, int64_t k) { return slices_bytes(plans(rows, k, n).most_slices, rows * k); }

aq_status launch_input_grad(const aq_matrix& dy, const aq_mx4& w, const aq_matrix& dx, void* ws, uint64_t ws_bytes, hipStream_t st) {
    const int64_t n = w.rows, k = w.cols, rows = dy.rows;
    const Plans all = plans(rows, k, n);
    const Plan p = all.of[type_of(dy.dtype)];
    if (!workspace_ok(ws, ws_bytes, slices_bytes(all.most_slices, rows * k))) return AQ_EINVAL;
    return with_dtype(dy.dtype, [&](auto t) {
        using T = decltype(t);
        const aq_status s = with_tile(p.s, [&](auto sc) {
            constexpr int S = decltype(sc)::value;
            auto go = [&](auto edge) {
                using A = DyCols<T, S, decltype(edge)::value>;
                constexpr int kSets = A::kSets;
                const A a{words_of<T>(dy)};
                using Weights = BlockRows<S, kSets, 4>;
                const Weights b{(const uint8_t*)w.d_codes, w.d_scales, blocks32(k), n};
                const int64_t bytes_per_t = 16 * blocks32(k);
                if (p.z > 1) return launch<A, Weights, float, S>(a, b, (float*)ws, k, rows * k, nullptr, rows, k, n, p, bytes_per_t, st);
                return launch<A, Weights, T, S>(a, b, (T*)dx.d, dx.ld, 0, nullptr, rows, k, n, p, bytes_per_t, st);
            };
            return any_pieces<T>(dy, true) ? go(std::true_type()) : go(std::false_type());
        });
        if (s != AQ_OK || p.z == 1) return s;
        return join((const float*)ws, p, rows, k, (T*)dx.d, dx.ld, nullptr, nullptr, st);
    });
}

}  // namespace aq
