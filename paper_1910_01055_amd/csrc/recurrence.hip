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

constexpr int kMostParts = 64;

template <class T, int V>
struct Units;  // V neighbouring values, as they lie in memory
template <>
struct Units<float, 1> {
    uint32_t w;
    __device__ __forceinline__ void load(const float* p) { w = *(const uint32_t AQ_GLOBAL*)p; }
    __device__ __forceinline__ void get(float (&v)[1]) const { v[0] = __uint_as_float(w); }
    static __device__ __forceinline__ void put(float* p, const float (&v)[1]) { *(float AQ_GLOBAL*)p = v[0]; }
};
template <>
struct Units<float, 2> {
    v2u w;
    __device__ __forceinline__ void load(const float* p) { w = *(const v2u_any AQ_GLOBAL*)p; }
    __device__ __forceinline__ void get(float (&v)[2]) const { v[0] = __uint_as_float(w[0]), v[1] = __uint_as_float(w[1]); }
    static __device__ __forceinline__ void put(float* p, const float (&v)[2]) {
        *(v2u_any AQ_GLOBAL*)p = v2u{__float_as_uint(v[0]), __float_as_uint(v[1])};
    }
};
template <class T>
struct Units<T, 1> {
    T w;
    __device__ __forceinline__ void load(const T* p) { w = *(const T AQ_GLOBAL*)p; }
    __device__ __forceinline__ void get(float (&v)[1]) const { v[0] = (float)w; }
    static __device__ __forceinline__ void put(T* p, const float (&v)[1]) { *(T AQ_GLOBAL*)p = (T)v[0]; }
};
template <class T>
struct Units<T, 2> {
    typedef T t2 __attribute__((ext_vector_type(2)));
    typedef uint32_t word __attribute__((aligned(2)));
    uint32_t w;
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
// (A, B) after (a, b): the map of both
__device__ __forceinline__ void then(float& a, float& b, float A, float B) {
    b = A < 0.0f ? B : fmaf(A, b, B);
    a = A < 0.0f || a < 0.0f ? -1.0f : A * a;
}
__device__ __forceinline__ float apply(float a, float b, float h) { return a < 0.0f ? b : fmaf(a, h, b); }

struct Rows {
    const int32_t* offsets;
    int64_t rows, count, cols;
    int parts;
};
// the rows of one lane's sequence that its workgroup takes
struct Span {
    int64_t begin, first, end, behind;  // of the sequence, of the part, behind the part, behind the sequence
    int64_t seq;
    int unit;
    bool active;
};
template <int V>
__device__ __forceinline__ Span span_of(const Rows& r, int part) {
    Span s;
    const int64_t across = r.cols / V, q = (int64_t)blockIdx.x * 64 + (threadIdx.x & 63);
    s.active = q < r.count * across;
    s.seq = s.active ? (r.count == 1 ? 0 : q / across) : 0;
    s.unit = s.active ? (int)(q - s.seq * across) * V : 0;
    if (r.offsets) {
        const int64_t a = r.offsets[s.seq], b = r.offsets[s.seq + 1];
        s.begin = a < 0 ? 0 : a > r.rows ? r.rows : a;
        s.behind = b < s.begin ? s.begin : b > r.rows ? r.rows : b;
    } else {
        const int64_t each = r.rows / r.count;
        s.begin = s.seq * each;
        s.behind = s.begin + each;
    }
    if (!s.active) s.behind = s.begin;
    const int64_t len = s.behind - s.begin;
    s.first = s.begin + len * part / r.parts;
    s.end = s.begin + len * (part + 1) / r.parts;
    return s;
}
__device__ __forceinline__ int64_t longest_of(int64_t n) {
    int m = (int)n;
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
            lds_barrier();
#pragma unroll
            for (int w = 0; w < W; ++w)
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    if (w == wave) in[v] = carry[v];
                    carry[v] = apply(ab[turn & 1][w][2 * v][lane], ab[turn & 1][w][2 * v + 1][lane], carry[v]);
                }
        }
    }
    static __device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
};

// where parts leave and find their (A, B): [part][A, B][count][cols]
__device__ __forceinline__ float* sum_at(float* sums, const Rows& r, int part, int which, const Span& s) {
    return sums + (((int64_t)part * 2 + which) * r.count + s.seq) * r.cols + s.unit;
}
template <int V>
__device__ __forceinline__ void carry_of_parts(float* sums, const Rows& r, int from, int to, int step, const Span& s, float (&carry)[V]) {
    for (int p = from; p != to; p += step)
#pragma unroll
        for (int v = 0; v < V; ++v) carry[v] = apply(sum_at(sums, r, p, 0, s)[v], sum_at(sums, r, p, 1, s)[v], carry[v]);
}

template <class T, int V, int R, int W, bool SUMS>
__global__ void __launch_bounds__(64 * W) k_recurrence(const T* __restrict__ z, int64_t ldz, const T* __restrict__ v, int64_t ldv, T* __restrict__ y,
                                                       int64_t ldy, const uint8_t* __restrict__ starts, const float* first, float* last, Rows rows,
                                                       float* __restrict__ sums) {
    __shared__ Exchange<V, W> exchange;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), part = blockIdx.y;
    const Span s = span_of<V>(rows, part);
    float carry[V], whole_a[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        carry[i] = !SUMS && first && s.active ? first[s.seq * rows.cols + s.unit + i] : 0.0f;
        whole_a[i] = 1.0f;
    }
    if constexpr (!SUMS)
        if (part && s.active) carry_of_parts(sums, rows, 0, part, 1, s, carry);
    const int64_t n = s.end - s.first, longest = longest_of(n);
    const int64_t safe = n > 0 ? s.first : 0;  // a row that exists
    const T *pz = z + s.unit, *pv = v + s.unit;
    int turn = 0;
    for (int64_t t0 = 0; t0 < longest; t0 += R * W, ++turn) {
        const int64_t mine = t0 + R * wave;
        const int left = n - mine < R ? (int)(n - mine) : R;
        Units<T, V> rz[R], rv[R];
        uint32_t cuts = 0;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t row = r < left ? s.first + mine + r : safe;
            rz[r].load(pz + row * ldz);
            rv[r].load(pv + row * ldv);
            if (starts) cuts |= (starts[row] != 0 ? 1u : 0u) << r;
        }
        float f[R][V], u[R][V], a[V], b[V];
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
                if (cuts >> r & 1) f[r][i] = -1.0f;
                if (r >= left) f[r][i] = 1.0f, u[r][i] = 0.0f;
                then(a[i], b[i], f[r][i], u[r][i]);
            }
        }
        float h[V];
        exchange.run(turn, wave, lane, a, b, carry, h);
        if constexpr (SUMS) {
            // carry began at 0, so that it is B; A of all wavefronts
            if constexpr (W == 1) {
#pragma unroll
                for (int i = 0; i < V; ++i) whole_a[i] = a[i] < 0.0f || whole_a[i] < 0.0f ? -1.0f : a[i] * whole_a[i];
            } else {
#pragma unroll
                for (int w = 0; w < W; ++w)
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const float aw = exchange.ab[turn & 1][w][2 * i][lane];
                        whole_a[i] = aw < 0.0f || whole_a[i] < 0.0f ? -1.0f : aw * whole_a[i];
                    }
            }
        } else {
#pragma unroll
            for (int r = 0; r < R; ++r) {
#pragma unroll
                for (int i = 0; i < V; ++i) h[i] = apply(f[r][i], u[r][i], h[i]);
                if (r < left) Units<T, V>::put(y + (s.first + mine + r) * ldy + s.unit, h);
            }
        }
    }
    if (wave != 0 || !s.active) return;
    if constexpr (SUMS) {
#pragma unroll
        for (int i = 0; i < V; ++i) sum_at(sums, rows, part, 0, s)[i] = whole_a[i], sum_at(sums, rows, part, 1, s)[i] = carry[i];
    } else if (last && part == rows.parts - 1) {
#pragma unroll
        for (int i = 0; i < V; ++i) last[s.seq * rows.cols + s.unit + i] = carry[i];
    }
}

// The same from the last row to the first: row r of a wavefront's run is the part's row n - 1 - (mine + r).
template <class T, int V, int R, int W, bool SUMS>
__global__ void __launch_bounds__(64 * W)
    k_recurrence_backward(const T* __restrict__ dy, int64_t lddy, const T* __restrict__ z, int64_t ldz, const T* __restrict__ v, int64_t ldv,
                          const T* __restrict__ y, int64_t ldy, const uint8_t* __restrict__ starts, const float* __restrict__ first,
                          const float* dlast, T* __restrict__ dz, int64_t lddz, T* __restrict__ dv, int64_t lddv, float* dfirst, Rows rows,
                          float* __restrict__ sums) {
    __shared__ Exchange<V, W> exchange;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), part = blockIdx.y;
    const Span s = span_of<V>(rows, part);
    float carry[V], whole_a[V], before[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        carry[i] = !SUMS && dlast && s.active ? dlast[s.seq * rows.cols + s.unit + i] : 0.0f;
        before[i] = !SUMS && first && s.active ? first[s.seq * rows.cols + s.unit + i] : 0.0f;
        whole_a[i] = 1.0f;
    }
    if constexpr (!SUMS)
        if (part != rows.parts - 1 && s.active) carry_of_parts(sums, rows, rows.parts - 1, part, -1, s, carry);
    const int64_t n = s.end - s.first, longest = longest_of(n);
    const int64_t safe = n > 0 ? s.first : 0;
    int turn = 0;
    for (int64_t t0 = 0; t0 < longest; t0 += R * W, ++turn) {
        const int64_t mine = t0 + R * wave;
        const int left = n - mine < R ? (int)(n - mine) : R;
        const int64_t top = s.end - 1 - mine;
        Units<T, V> rz[R], rd[R], rv[SUMS ? 1 : R], ry[SUMS ? 1 : R];
        uint32_t cuts = 0;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t row = r < left ? top - r : safe;
            rz[r].load(z + row * ldz + s.unit);
            rd[r].load(dy + row * lddy + s.unit);
            if constexpr (!SUMS) {
                rv[r].load(v + row * ldv + s.unit);
                ry[r].load(y + (row > s.begin ? row - 1 : row) * ldy + s.unit);
            }
            if (starts) cuts |= (starts[row] != 0 ? 1u : 0u) << r;
        }
        float f[R][V], rest[R][V], d[R][V], a[V], b[V];
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
                float A = f[r][i], B = f[r][i] * d[r][i];
                if (cuts >> r & 1) A = -1.0f, B = 0.0f;
                if (r >= left) A = 1.0f, B = 0.0f;
                then(a[i], b[i], A, B);
            }
        }
        float G[V];
        exchange.run(turn, wave, lane, a, b, carry, G);
        if constexpr (SUMS) {
            if constexpr (W == 1) {
#pragma unroll
                for (int i = 0; i < V; ++i) whole_a[i] = a[i] < 0.0f || whole_a[i] < 0.0f ? -1.0f : a[i] * whole_a[i];
            } else {
#pragma unroll
                for (int w = 0; w < W; ++w)
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const float aw = exchange.ab[turn & 1][w][2 * i][lane];
                        whole_a[i] = aw < 0.0f || whole_a[i] < 0.0f ? -1.0f : aw * whole_a[i];
                    }
            }
        } else {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if (r >= left) break;
                const int64_t row = top - r;
                float x[V], h[V], oz[V], ov[V];
                rv[r].get(x);
                ry[r].get(h);
                const bool cut = cuts >> r & 1;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float hb = cut ? 0.0f : row > s.begin ? h[i] : before[i];
                    const float g = d[r][i] + G[i];
                    ov[i] = g * rest[r][i];
                    oz[i] = ov[i] * f[r][i] * (hb - x[i]);
                    G[i] = cut ? 0.0f : f[r][i] * g;
                }
                Units<T, V>::put(dv + row * lddv + s.unit, ov);
                Units<T, V>::put(dz + row * lddz + s.unit, oz);
            }
        }
    }
    if (wave != 0 || !s.active) return;
    if constexpr (SUMS) {
#pragma unroll
        for (int i = 0; i < V; ++i) sum_at(sums, rows, part, 0, s)[i] = whole_a[i], sum_at(sums, rows, part, 1, s)[i] = carry[i];
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

// parts of a sequence
int parts_of(int64_t rows, int64_t count, int64_t cols) {
    const int64_t groups = (count * cols + 127) / 128, mean = rows / count;
    int64_t parts = 1024 / (groups > 0 ? groups : 1);
    if (parts > mean / 256) parts = mean / 256;
    return parts < 2 ? 1 : parts > kMostParts ? kMostParts : (int)parts;
}
int waves_of(int64_t steps, int rows) { return steps <= rows ? 1 : steps <= 2 * rows ? 2 : steps <= 4 * rows ? 4 : 8; }
template <int N>
using Int = std::integral_constant<int, N>;
template <class Go>
aq_status with_waves(int w, Go&& go) {
    return w == 1 ? go(Int<1>()) : w == 2 ? go(Int<2>()) : w == 4 ? go(Int<4>()) : go(Int<8>());
}
template <class Go>
aq_status with_units(int64_t cols, Go&& go) {
    return cols % 2 == 0 ? go(Int<2>()) : go(Int<1>());
}
aq_status launched() { return hip_failed(hipGetLastError()) ? AQ_EHIP : AQ_OK; }

}  // namespace

int64_t recurrence_workspace(int64_t rows, int64_t count, int64_t cols) {
    const int64_t parts = count > 0 ? parts_of(rows, count, cols) : 1;
    return parts < 2 ? 0 : parts * 2 * count * cols * (int64_t)sizeof(float);
}

aq_status launch_recurrence_forward(const aq_matrix& z, const aq_matrix& v, const int32_t* offsets, int64_t count, const uint8_t* starts,
                                    const float* first, const aq_matrix& y, float* last, float* ws, hipStream_t st) {
    constexpr int R = 16;
    const int parts = parts_of(z.rows, count, z.cols);
    const Rows rows{offsets, z.rows, count, z.cols, parts};
    return with_dtype(z.dtype, [&](auto t) {
        using T = decltype(t);
        return with_units(z.cols, [&](auto units) {
            constexpr int V = decltype(units)::value;
            return with_waves(waves_of(z.rows / count / parts, R), [&](auto waves) {
                constexpr int W = decltype(waves)::value;
                const dim3 grid((uint32_t)((count * (z.cols / V) + 63) / 64), parts);
                if (parts > 1)
                    k_recurrence<T, V, R, W, true><<<grid, 64 * W, 0, st>>>((const T*)z.d, z.ld, (const T*)v.d, v.ld, (T*)y.d, y.ld, starts, first,
                                                                            last, rows, ws);
                k_recurrence<T, V, R, W, false><<<grid, 64 * W, 0, st>>>((const T*)z.d, z.ld, (const T*)v.d, v.ld, (T*)y.d, y.ld, starts, first, last,
                                                                         rows, ws);
                return launched();
            });
        });
    });
}

aq_status launch_recurrence_backward(const aq_matrix& dy, const float* dlast, const aq_matrix& z, const aq_matrix& v, const aq_matrix& y,
                                     const int32_t* offsets, int64_t count, const uint8_t* starts, const float* first, const aq_matrix& dz,
                                     const aq_matrix& dv, float* dfirst, float* ws, hipStream_t st) {
    constexpr int R = 8;
    const int parts = parts_of(z.rows, count, z.cols);
    const Rows rows{offsets, z.rows, count, z.cols, parts};
    return with_dtype(z.dtype, [&](auto t) {
        using T = decltype(t);
        return with_units(z.cols, [&](auto units) {
            constexpr int V = decltype(units)::value;
            return with_waves(waves_of(z.rows / count / parts, R), [&](auto waves) {
                constexpr int W = decltype(waves)::value;
                const dim3 grid((uint32_t)((count * (z.cols / V) + 63) / 64), parts);
                auto run = [&](auto kernel) {
                    kernel<<<grid, 64 * W, 0, st>>>((const T*)dy.d, dy.ld, (const T*)z.d, z.ld, (const T*)v.d, v.ld, (const T*)y.d, y.ld, starts, first,
                                                    dlast, (T*)dz.d, dz.ld, (T*)dv.d, dv.ld, dfirst, rows, ws);
                };
                if (parts > 1) run(k_recurrence_backward<T, V, R, W, true>);
                run(k_recurrence_backward<T, V, R, W, false>);
                return launched();
            });
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
