// A gated linear recurrence over sequences of rows, unit by unit, its gradients and its single step.
//
//   h_t = k_t h_{t-1} + (1 - f_t) v_t,  f = sigmoid(z),  k_t = f_t, or 0 where an episode starts
//   G_t = k_t (dy_t + G_{t+1}) from the last row to the first;  g_t = dy_t + G_{t+1}:  dv = (1 - f) g,  dz = g (k_t h_{t-1} / f_t - v) f (1 - f)
//
// Bound by memory: three values a step and unit forward, six backward.  Steps are affine maps h -> A h + B, whose composition is one
// again: a run of rows is summed up by (A, B), and runs side by side need each other's (A, B) only.  A lane holds V neighbouring units
// of one sequence (pairs of units are numbered over all sequences, so that no lane idles where units are few), a wavefront R rows of them
// at a time in registers; W wavefronts take R rows each, exchange (A, B) through LDS and go over their rows once more, from the state that
// theirs begin with, without another read.  Where sequences and units are too few to fill the chip, every sequence is cut into as
// many parts as it takes, in proportion to its length, and a launch in front of this one leaves the parts' (A, B).
// The state and (A, B) are fp32; a start that cuts a run is kept as A = -1, which no product gives: a NaN in front of it ends there.
#include "learner.hpp"
#include "learner_device.hpp"

namespace aq {
namespace {

constexpr int64_t kMostParts = 256;  // of a sequence

template <class T, int V>
struct Units;  // V neighbouring values, as they lie in memory
template <class T>
constexpr uint32_t kInfinities = std::is_same<T, float>::value ? 0x7f800000u : std::is_same<T, bf16_t>::value ? 0x7f807f80u : 0x7c007c00u;
template <>
struct Units<float, 1> {
    uint32_t w;
    __device__ __forceinline__ void set(uint32_t two) { w = two; }
    __device__ __forceinline__ void load(const float* p) { w = *(const uint32_t AQ_GLOBAL*)p; }
    __device__ __forceinline__ void get(float (&v)[1]) const { v[0] = __uint_as_float(w); }
    static __device__ __forceinline__ void put(float* p, const float (&v)[1]) { *(float AQ_GLOBAL*)p = v[0]; }
};
template <>
struct Units<float, 2> {
    v2u w;
    __device__ __forceinline__ void set(uint32_t two) { w = v2u{two, two}; }
    __device__ __forceinline__ void load(const float* p) { w = *(const v2u_any AQ_GLOBAL*)p; }
    __device__ __forceinline__ void get(float (&v)[2]) const { v[0] = __uint_as_float(w[0]), v[1] = __uint_as_float(w[1]); }
    static __device__ __forceinline__ void put(float* p, const float (&v)[2]) {
        *(v2u_any AQ_GLOBAL*)p = v2u{__float_as_uint(v[0]), __float_as_uint(v[1])};
    }
};
template <class T>
struct Units<T, 1> {
    T w;
    __device__ __forceinline__ void set(uint32_t two) { w = __builtin_bit_cast(T, (uint16_t)two); }
    __device__ __forceinline__ void load(const T* p) { w = *(const T AQ_GLOBAL*)p; }
    __device__ __forceinline__ void get(float (&v)[1]) const { v[0] = (float)w; }
    static __device__ __forceinline__ void put(T* p, const float (&v)[1]) { *(T AQ_GLOBAL*)p = (T)v[0]; }
};
template <class T>
struct Units<T, 2> {
    typedef T t2 __attribute__((ext_vector_type(2)));
    typedef uint32_t word __attribute__((aligned(2)));
    uint32_t w;
    __device__ __forceinline__ void set(uint32_t two) { w = two; }
    __device__ __forceinline__ void load(const T* p) { w = *(const word AQ_GLOBAL*)p; }
    __device__ __forceinline__ void get(float (&v)[2]) const {
        if constexpr (std::is_same<T, bf16_t>::value) {
            v[0] = __uint_as_float(w << 16), v[1] = __uint_as_float(w & 0xffff0000u);
        } else {
            const t2 h = __builtin_bit_cast(t2, w);
            v[0] = (float)h[0], v[1] = (float)h[1];
        }
    }
    static __device__ __forceinline__ void put(T* p, const float (&v)[2]) {
        *(word AQ_GLOBAL*)p = __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f32{v[0], v[1]}), t2));
    }
};

// sigmoid(z) and sigmoid(-z), neither as a difference from 1
__device__ __forceinline__ void gates(float z, float& f, float& rest) {
    const float e = __builtin_amdgcn_exp2f(-1.44269504f * fabsf(z));
    const float large = __builtin_amdgcn_rcpf(1.0f + e), small = e * large;
    f = z >= 0.0f ? large : small;
    rest = z >= 0.0f ? small : large;
}
// the same value to the program, another one to the compiler, which else keeps every comparison with it for the second pass in registers
__device__ __forceinline__ uint32_t anew(uint32_t v) {
    asm volatile("" : "+v"(v));
    return v;
}
__device__ __forceinline__ float apply(float a, float b, float h) { return a < 0.0f ? b : fmaf(a, h, b); }

struct Rows {
    const int32_t* offsets;
    int64_t rows, cols, each;  // each: rows of a sequence, without offsets
    int32_t count, across;     // sequences; lanes to one
    int32_t parts, least;      // most parts of a sequence, and the least rows of one
};
// Rows of one lane's sequence that its workgroup takes.  A sequence has as many parts as its rows fill, so that short ones need no sums;
// its parts' sums lie from slot begin / least + (its number) on, which no other one's reach.
struct Span {
    int64_t begin, first, behind;  // of the sequence; of the part; behind the sequence
    int n, parts;                  // rows of the part; parts of the sequence
    int seq, unit;
    bool active;                   // has such a part
};
template <int V>
__device__ __forceinline__ Span span_of(const Rows& r, int part) {
    Span s;
    const uint32_t q = blockIdx.x * 64 + (threadIdx.x & 63);
    s.seq = (int)(q / (uint32_t)r.across);
    s.active = s.seq < r.count;
    if (!s.active) s.seq = 0;
    s.unit = (int)(q % (uint32_t)r.across) * V;
    if (V > 1 && s.unit > (int)r.cols - V) s.unit = (int)r.cols - V;  // (units that two lanes have are the same in both)
    if (r.offsets) {
        const int64_t a = r.offsets[s.seq], b = r.offsets[s.seq + 1];
        s.begin = a < 0 ? 0 : a > r.rows ? r.rows : a;
        s.behind = b < s.begin ? s.begin : b > r.rows ? r.rows : b;
    } else {
        s.begin = s.seq * r.each;
        s.behind = s.begin + r.each;
    }
    const int len = (int)(s.behind - s.begin);
    s.first = s.begin;
    s.n = len;
    s.parts = 1;
    if (r.parts > 1) {
        s.parts = len / r.least;
        s.parts = s.parts < 1 ? 1 : s.parts > r.parts ? r.parts : s.parts;
        const int each = (len + s.parts - 1) / s.parts;
        s.active = s.active && part < s.parts;
        s.first = s.begin + (int64_t)each * part;
        s.n = s.first + each < s.behind ? each : (int)(s.behind - s.first);
        if (s.n < 0) s.n = 0, s.first = s.behind;
    }
    if (!s.active) s.n = 0;
    return s;
}
__device__ __forceinline__ int longest_of(int m) {
#pragma unroll
    for (int k = 32; k; k >>= 1) {
        const int o = __shfl_xor(m, k);
        m = o > m ? o : m;
    }
    return __builtin_amdgcn_readfirstlane(m);
}

// Exchange of W wavefronts' (A, B) of the same lanes: `in` gets the state in front of this wavefront's rows, `carry` that behind all.
template <int V, int W>
struct Exchange {
    float ab[W > 1 ? 2 : 1][W > 1 ? W : 1][2 * V][64];
    __device__ __forceinline__ void run(int turn, int wave, int lane, const float (&a)[V], const float (&b)[V], float (&carry)[V], float (&in)[V]) {
        if constexpr (W == 1) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                in[v] = carry[v];
                carry[v] = apply(a[v], b[v], carry[v]);
            }
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) ab[turn & 1][wave][2 * v][lane] = a[v], ab[turn & 1][wave][2 * v + 1][lane] = b[v];
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");  // (loads from memory stay in flight)
#pragma unroll
            for (int w = 0; w < W; ++w)
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    if (w == wave) in[v] = carry[v];
                    carry[v] = apply(ab[turn & 1][w][2 * v][lane], ab[turn & 1][w][2 * v + 1][lane], carry[v]);
                }
        }
    }
    // A of all wavefronts' rows behind `whole`
    __device__ __forceinline__ void extend(int turn, int lane, const float (&a)[V], float (&whole)[V]) const {
#pragma unroll
        for (int w = 0; w < W; ++w)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float x = W == 1 ? a[v] : ab[turn & 1][w][2 * v][lane];
                whole[v] = x < 0.0f || whole[v] < 0.0f ? -1.0f : x * whole[v];
            }
    }
};

// where parts leave and find their (A, B): [slot][A, B][cols]
__device__ __forceinline__ float* sum_at(float* sums, const Rows& r, int part, int which, const Span& s) {
    return sums + ((s.begin / r.least + s.seq + part) * 2 + which) * r.cols + s.unit;
}
// The state in front of a part, from the sums of the parts `from`, from + step .. (`many` of them, those below `parts` of which exist): each
// wavefront joins a run of them, four on their way at a time.
template <int V, int W>
__device__ __forceinline__ void carry_of_parts(Exchange<V, W>& exchange, float* sums, const Rows& r, int from, int many, int step, const Span& s,
                                               int wave, int lane, float (&carry)[V]) {
    const int each = (many + W - 1) / W, first = wave * each, end = first + each < many ? first + each : many;
    float a[V], b[V], unused[V];
#pragma unroll
    for (int v = 0; v < V; ++v) a[v] = 1.0f, b[v] = 0.0f;
    for (int k = first; k < end; k += 4) {
        float A[4][V], B[4][V];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int p = from + (k + i) * step;
            const bool there = k + i < end && p < s.parts && s.active;
#pragma unroll
            for (int v = 0; v < V; ++v) A[i][v] = there ? sum_at(sums, r, p, 0, s)[v] : 1.0f, B[i][v] = there ? sum_at(sums, r, p, 1, s)[v] : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                b[v] = apply(A[i][v], B[i][v], b[v]);
                a[v] = A[i][v] < 0.0f || a[v] < 0.0f ? -1.0f : A[i][v] * a[v];
            }
    }
    exchange.run(1, wave, lane, a, b, carry, unused);
}

// Which of the R rows from `row` on start an episode, of those below `rows`.
template <int R>
struct Starts {
    typedef uint32_t words __attribute__((ext_vector_type(R / 4), aligned(1)));
    words w;
    __device__ __forceinline__ void load(const uint8_t* __restrict__ starts, int64_t row, int64_t rows) {
        if (row >= 0 && row + R <= rows) {
            w = *(const words AQ_GLOBAL*)(starts + row);
        } else {
#pragma unroll
            for (int i = 0; i < R / 4; ++i) w[i] = 0;
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (row + r >= 0 && row + r < rows) w[r / 4] |= (uint32_t)starts[row + r] << (8 * (r & 3));
        }
    }
    __device__ __forceinline__ uint32_t bits() const {  // bit r for row + r
        uint32_t cuts = 0;
#pragma unroll
        for (int i = 0; i < R / 4; ++i) {
            // the upper bit of each byte that is not 0, then the four of them side by side
            const uint32_t x = w[i], some = (((x & 0x7f7f7f7fu) + 0x7f7f7f7fu) | x) >> 7 & 0x01010101u;
            cuts |= (some * 0x10204080u >> 28) << (4 * i);
        }
        return cuts;
    }
};

template <class T, int V, int R, int W, bool SUMS, bool STARTS>
__global__ void __launch_bounds__(64 * W) k_recurrence(const T* __restrict__ z, int64_t ldz, const T* __restrict__ v, int64_t ldv, T* __restrict__ y,
                                                       int64_t ldy, const uint8_t* __restrict__ starts, const float* first, float* last, Rows rows,
                                                       float* __restrict__ sums) {
    __shared__ Exchange<V, W> exchange;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), part = blockIdx.y;
    const Span s = span_of<V>(rows, part);
    const bool summed = SUMS ? s.active && s.parts > 1 && part < s.parts - 1 : s.active;  // (the last part's sums reach nothing)
    const int n = summed ? s.n : 0, longest = longest_of(n);
    float carry[V], whole[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        carry[i] = !SUMS && first && s.active ? first[s.seq * rows.cols + s.unit + i] : 0.0f;
        whole[i] = 1.0f;
    }
    if constexpr (!SUMS)
        if (part) carry_of_parts(exchange, sums, rows, 0, part, 1, s, wave, lane, carry);
    Units<T, V> rz[R], rv[R];
    Starts<R> rs;
    auto left_of = [&](int t0) __attribute__((always_inline)) { return n - t0 - R * wave < R ? n - t0 - R * wave : R; };
    auto row_of = [&](int t0, int left) __attribute__((always_inline)) { return n > 0 ? s.first + (left > 0 ? t0 + R * wave : 0) : 0; };  // (one that exists)
    auto load = [&](int t0) __attribute__((always_inline)) {
        const int left = left_of(t0), most = longest - t0 - R * wave;  // rows of this lane's, and of some lane's
        const int64_t row = row_of(t0, left);
        const T *pz = z + row * ldz + s.unit, *pv = v + row * ldv + s.unit;
        if (__all(left == R)) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                rz[r].load(pz + r * ldz);
                rv[r].load(pv + r * ldv);
            }
        } else {
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (r < most) {
                    rz[r].load(r < left ? pz + r * ldz : pz);
                    rv[r].load(r < left ? pv + r * ldv : pv);
                }
        }
        if (STARTS && left > 0) rs.load(starts, row, rows.rows);
    };
    int turn = 0;
    if (longest > 0) load(0);
    for (int t0 = 0; t0 < longest; t0 += R * W, ++turn) {
        const int left = left_of(t0);
        const bool full = __all(left == R);
        if (!full) {  // rows that are not there change nothing: f = 1
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (r >= left) rz[r].set(kInfinities<T>), rv[r].set(0);
        }
        uint32_t cuts = STARTS && left > 0 ? rs.bits() & ((2u << (left - 1)) - 1) : 0u;
        float f[R][V], u[R][V], a[V], b[V], h[V];
#pragma unroll
        for (int i = 0; i < V; ++i) a[i] = 1.0f, b[i] = 0.0f;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float x[V], rest;
            rz[r].get(f[r]);
            rv[r].get(x);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                gates(f[r][i], f[r][i], rest);
                u[r][i] = rest * x[i];
                a[i] *= f[r][i];
                b[i] = STARTS && (cuts >> r & 1) ? u[r][i] : fmaf(f[r][i], b[i], u[r][i]);
            }
        }
        if constexpr (STARTS) {
#pragma unroll
            for (int i = 0; i < V; ++i) a[i] = cuts ? -1.0f : a[i];
            cuts = anew(cuts);
        }
        if (t0 + R * W < longest) load(t0 + R * W);  // on its way during the exchange and the second pass
        exchange.run(turn, wave, lane, a, b, carry, h);
        if constexpr (SUMS) {
            exchange.extend(turn, lane, a, whole);
        } else {
            T* const py = y + row_of(t0, left) * ldy + s.unit;
            const int stored = full ? R : (int)anew(left);
#pragma unroll
            for (int r = 0; r < R; ++r) {
#pragma unroll
                for (int i = 0; i < V; ++i) h[i] = STARTS && (cuts >> r & 1) ? u[r][i] : fmaf(f[r][i], h[i], u[r][i]);
                if (r < stored) Units<T, V>::put(py + r * ldy, h);
            }
        }
    }
    if (wave != 0 || !summed) return;
    if constexpr (SUMS) {
#pragma unroll
        for (int i = 0; i < V; ++i) sum_at(sums, rows, part, 0, s)[i] = whole[i], sum_at(sums, rows, part, 1, s)[i] = carry[i];
    } else if (last && part == s.parts - 1) {
#pragma unroll
        for (int i = 0; i < V; ++i) last[s.seq * rows.cols + s.unit + i] = carry[i];
    }
}

// The same from the last row to the first: row r of a wavefront's run is the part's row n - 1 - (mine + r).
template <class T, int V, int R, int W, bool SUMS, bool STARTS>
__global__ void __launch_bounds__(64 * W)
    k_recurrence_backward(const T* __restrict__ dy, int64_t lddy, const T* __restrict__ z, int64_t ldz, const T* __restrict__ v, int64_t ldv,
                          const T* __restrict__ y, int64_t ldy, const uint8_t* __restrict__ starts, const float* __restrict__ first,
                          const float* dlast, T* __restrict__ dz, int64_t lddz, T* __restrict__ dv, int64_t lddv, float* dfirst, Rows rows,
                          float* __restrict__ sums) {
    __shared__ Exchange<V, W> exchange;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), part = blockIdx.y;
    const Span s = span_of<V>(rows, part);
    const bool summed = SUMS ? s.active && part > 0 : s.active;  // (the first part's sums reach nothing)
    const int n = summed ? s.n : 0, longest = longest_of(n);
    float carry[V], whole[V], before[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        carry[i] = !SUMS && dlast && s.active ? dlast[s.seq * rows.cols + s.unit + i] : 0.0f;
        before[i] = !SUMS && first && s.active ? first[s.seq * rows.cols + s.unit + i] : 0.0f;
        whole[i] = 1.0f;
    }
    if constexpr (!SUMS) {
        const int behind = longest_of(s.active ? s.parts - 1 - part : 0);
        if (behind) carry_of_parts(exchange, sums, rows, part + behind, behind, -1, s, wave, lane, carry);
    }
    Units<T, V> rz[R], rd[R], rv[SUMS ? 1 : R], ry[SUMS ? 1 : R];
    Starts<R> rs;
    auto left_of = [&](int t0) __attribute__((always_inline)) { return n - t0 - R * wave < R ? n - t0 - R * wave : R; };
    auto top_of = [&](int t0, int left) __attribute__((always_inline)) {  // the run's last row, or one that exists
        return n > 0 ? s.first + (left > 0 ? n - 1 - t0 - R * wave : 0) : 0;
    };
    auto full_of = [&](int64_t top, int left) __attribute__((always_inline)) { return __all(left == R && top - R >= s.begin); };
    auto load = [&](int t0) __attribute__((always_inline)) {
        const int left = left_of(t0), most = longest - t0 - R * wave;
        const int64_t top = top_of(t0, left);
        const T *pz = z + top * ldz + s.unit, *pd = dy + top * lddy + s.unit;
        if (full_of(top, left)) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                rz[r].load(pz - r * ldz);
                rd[r].load(pd - r * lddy);
            }
        } else {
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (r < most) {
                    rz[r].load(r < left ? pz - r * ldz : pz);
                    rd[r].load(r < left ? pd - r * lddy : pd);
                }
        }
        if (STARTS && left > 0) rs.load(starts, top - (R - 1), rows.rows);
    };
    auto load_second = [&](int t0) __attribute__((always_inline)) {  // what the second pass reads
        const int left = left_of(t0), most = longest - t0 - R * wave;
        const int64_t top = top_of(t0, left);
        const T *pv = v + top * ldv + s.unit, *py = y + top * ldy + s.unit;
        if (full_of(top, left)) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                rv[r].load(pv - r * ldv);
                ry[r].load(py - (r + 1) * ldy);
            }
        } else {
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (r < most) {
                    rv[r].load(r < left ? pv - r * ldv : pv);
                    ry[r].load(r < left && top - r > s.begin ? py - (r + 1) * ldy : py);
                }
        }
    };
    int turn = 0;
    if (longest > 0) {
        load(0);
        if constexpr (!SUMS) load_second(0);
    }
    for (int t0 = 0; t0 < longest; t0 += R * W, ++turn) {
        const int left = left_of(t0);
        const int64_t top = top_of(t0, left);
        const bool full = full_of(top, left);
        if (!full) {
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (r >= left) rz[r].set(kInfinities<T>), rd[r].set(0);
        }
        uint32_t cuts = 0;  // bit R - 1 - r for row top - r
        if (STARTS && left > 0) cuts = rs.bits() >> (R - left) << (R - left);
        float f[R][V], rest[R][V], d[R][V], a[V], b[V], G[V];
#pragma unroll
        for (int i = 0; i < V; ++i) a[i] = 1.0f, b[i] = 0.0f;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            rz[r].get(f[r]);
            rd[r].get(d[r]);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                gates(f[r][i], f[r][i], rest[r][i]);
                // G = k (dy + G): a cut leaves zero, whatever came
                a[i] *= f[r][i];
                b[i] = STARTS && (cuts >> (R - 1 - r) & 1) ? 0.0f : f[r][i] * (d[r][i] + b[i]);
            }
        }
        if constexpr (STARTS) {
#pragma unroll
            for (int i = 0; i < V; ++i) a[i] = cuts ? -1.0f : a[i];
            cuts = anew(cuts);
        }
        if (t0 + R * W < longest) load(t0 + R * W);
        exchange.run(turn, wave, lane, a, b, carry, G);
        if constexpr (SUMS) {
            exchange.extend(turn, lane, a, whole);
        } else {
            T *const pdz = dz + top * lddz + s.unit, *const pdv = dv + top * lddv + s.unit;
            const int stored = full ? R : (int)anew(left), inside = full ? R : (int)(top - s.begin < R ? top - s.begin : R);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float x[V], h[V], oz[V], ov[V];
                rv[r].get(x);
                ry[r].get(h);
                const bool cut = STARTS && (cuts >> (R - 1 - r) & 1), has = r < inside;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float hb = cut ? 0.0f : has ? h[i] : before[i];
                    const float g = d[r][i] + G[i];
                    ov[i] = g * rest[r][i];
                    oz[i] = ov[i] * f[r][i] * (hb - x[i]);
                    G[i] = cut ? 0.0f : f[r][i] * g;
                }
                if (r < stored) {
                    Units<T, V>::put(pdv - r * lddv, ov);
                    Units<T, V>::put(pdz - r * lddz, oz);
                }
            }
            if (t0 + R * W < longest) load_second(t0 + R * W);
        }
    }
    if (wave != 0 || !summed) return;
    if constexpr (SUMS) {
#pragma unroll
        for (int i = 0; i < V; ++i) sum_at(sums, rows, part, 0, s)[i] = whole[i], sum_at(sums, rows, part, 1, s)[i] = carry[i];
    } else if (dfirst && part == 0) {
#pragma unroll
        for (int i = 0; i < V; ++i) dfirst[s.seq * rows.cols + s.unit + i] = carry[i];
    }
}

// One step of `rows` memories: eight units to a thread.
template <class T>
__global__ void __launch_bounds__(256) k_recurrence_step(const T* __restrict__ z, int64_t ldz, const T* __restrict__ v, int64_t ldv,
                                                         const uint8_t* __restrict__ starts, float* __restrict__ state, T* __restrict__ y, int64_t ldy,
                                                         int64_t rows, int cols) {
    const int64_t across = (cols + 7) / 8, step = (int64_t)gridDim.x * 256;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * across; i += step) {
        const int64_t row = i / across;
        const int unit = (int)(i - row * across) * 8, n = cols - unit;
        Piece<T> pz, pv, py;
        Piece<float> ps;
        pz.load(z + row * ldz + unit, n);
        pv.load(v + row * ldv + unit, n);
        ps.load(state + row * cols + unit, n);
        const bool cut = starts && starts[row];
        float a[8], x[8], h[8];
        pz.get(a);
        pv.get(x);
        ps.get(h);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float f, rest;
            gates(a[j], f, rest);
            h[j] = cut ? rest * x[j] : fmaf(f, h[j], rest * x[j]);
        }
        ps.set(h);
        ps.store(state + row * cols + unit, n);
        if (y) {
            py.set(h);
            py.store(y + row * ldy + unit, n);
        }
    }
}

// How sequences are cut: into parts of at least `least` rows.
struct Cut {
    int64_t parts, least;
};
Cut cut_of(int64_t rows, int64_t count, int64_t cols) {
    const int64_t across = cols > 1 ? (cols + 1) / 2 : 1, groups = (count * across + 63) / 64, mean = rows / count;
    const int64_t want = 1024 / groups;  // parts of each sequence that fill the chip
    int64_t least = mean < 1024 ? (mean < 256 ? 1024 : 4 * mean) : want > 1 ? mean / want : 4 * mean;
    if (least < 256) least = 256;
    int64_t parts = 8192 / groups;
    if (parts > kMostParts) parts = kMostParts;
    if (parts > rows / least) parts = rows / least;
    return {parts < 1 ? 1 : parts, least};
}
int waves_of(int64_t steps, int rows) { return steps <= rows ? 1 : steps <= 2 * rows ? 2 : steps <= 4 * rows ? 4 : 8; }
template <int N>
using Int = std::integral_constant<int, N>;
// calls go(units of a lane, wavefronts of a workgroup)
template <class Go>
aq_status with_form(int64_t cols, int waves, Go&& go) {
    auto by = [&](auto units) { return waves == 1 ? go(units, Int<1>()) : waves == 2 ? go(units, Int<2>()) : waves == 4 ? go(units, Int<4>()) : go(units, Int<8>()); };
    return cols > 1 ? by(Int<2>()) : by(Int<1>());
}
aq_status launched() { return hip_failed(hipGetLastError()) ? AQ_EHIP : AQ_OK; }
Rows rows_of(const int32_t* offsets, int64_t rows, int64_t count, int64_t cols) {
    const Cut cut = cut_of(rows, count, cols);
    const int64_t each = rows / count, parts = offsets || cut.parts * cut.least <= each ? cut.parts : each / cut.least;
    return {offsets, rows, cols, each, (int32_t)count, (int32_t)(cols > 1 ? (cols + 1) / 2 : 1), (int32_t)(parts < 1 ? 1 : parts), (int32_t)cut.least};
}
dim3 grid_of(const Rows& r) { return dim3((uint32_t)(((int64_t)r.count * r.across + 63) / 64), r.parts); }

}  // namespace

int64_t recurrence_workspace(int64_t rows, int64_t count, int64_t cols) {
    if (count < 1) return 0;
    const Cut cut = cut_of(rows, count, cols);
    return cut.parts < 2 ? 0 : (rows / cut.least + count + 1) * 2 * cols * (int64_t)sizeof(float);
}

aq_status launch_recurrence_forward(const aq_matrix& z, const aq_matrix& v, const int32_t* offsets, int64_t count, const uint8_t* starts,
                                    const float* first, const aq_matrix& y, float* last, float* ws, hipStream_t st) {
    constexpr int R = 16;
    const Rows rows = rows_of(offsets, z.rows, count, z.cols);
    const int64_t steps = rows.parts > 1 && rows.least < rows.each ? rows.least : rows.each;
    return with_dtype(z.dtype, [&](auto t) {
        using T = decltype(t);
        return with_form(z.cols, waves_of(steps, R), [&](auto units, auto waves) {
            constexpr int V = decltype(units)::value, W = decltype(waves)::value;
            auto run = [&](auto kernel) {
                kernel<<<grid_of(rows), 64 * W, 0, st>>>((const T*)z.d, z.ld, (const T*)v.d, v.ld, (T*)y.d, y.ld, starts, first, last, rows, ws);
            };
            if (starts) {
                if (rows.parts > 1) run(k_recurrence<T, V, R, W, true, true>);
                run(k_recurrence<T, V, R, W, false, true>);
            } else {
                if (rows.parts > 1) run(k_recurrence<T, V, R, W, true, false>);
                run(k_recurrence<T, V, R, W, false, false>);
            }
            return launched();
        });
    });
}

aq_status launch_recurrence_backward(const aq_matrix& dy, const float* dlast, const aq_matrix& z, const aq_matrix& v, const aq_matrix& y,
                                     const int32_t* offsets, int64_t count, const uint8_t* starts, const float* first, const aq_matrix& dz,
                                     const aq_matrix& dv, float* dfirst, float* ws, hipStream_t st) {
    constexpr int R = 8;
    const Rows rows = rows_of(offsets, z.rows, count, z.cols);
    const int64_t steps = rows.parts > 1 && rows.least < rows.each ? rows.least : rows.each;
    return with_dtype(z.dtype, [&](auto t) {
        using T = decltype(t);
        return with_form(z.cols, waves_of(steps, R), [&](auto units, auto waves) {
            constexpr int V = decltype(units)::value, W = decltype(waves)::value;
            auto run = [&](auto kernel) {
                kernel<<<grid_of(rows), 64 * W, 0, st>>>((const T*)dy.d, dy.ld, (const T*)z.d, z.ld, (const T*)v.d, v.ld, (const T*)y.d, y.ld, starts, first,
                                                         dlast, (T*)dz.d, dz.ld, (T*)dv.d, dv.ld, dfirst, rows, ws);
            };
            if (starts) {
                if (rows.parts > 1) run(k_recurrence_backward<T, V, R, W, true, true>);
                run(k_recurrence_backward<T, V, R, W, false, true>);
            } else {
                if (rows.parts > 1) run(k_recurrence_backward<T, V, R, W, true, false>);
                run(k_recurrence_backward<T, V, R, W, false, false>);
            }
            return launched();
        });
    });
}

aq_status launch_recurrence_step(const aq_matrix& z, const aq_matrix& v, const uint8_t* starts, float* state, const aq_matrix* y, hipStream_t st) {
    const int64_t pieces = z.rows * ((z.cols + 7) / 8), groups = (pieces + 255) / 256;
    return with_dtype(z.dtype, [&](auto t) {
        using T = decltype(t);
        k_recurrence_step<T><<<groups < 16384 ? (uint32_t)groups : 16384u, 256, 0, st>>>((const T*)z.d, z.ld, (const T*)v.d, v.ld, starts, state,
                                                                                         y ? (T*)y->d : nullptr, y ? y->ld : 0, z.rows, (int)z.cols);
        return launched();
    });
}

}  // namespace aq
