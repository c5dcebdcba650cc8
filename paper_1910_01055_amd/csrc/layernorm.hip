// LayerNorm and its gradients over rows of up to 16384 values, one pass over the data each.
//
//   y = (x - mean) rstd gamma + beta          dx = rstd (g - mean_row(g) - h mean_row(g h)),  g = dy gamma,  h = (x - mean) rstd
//   rstd = 1 / sqrt(var + eps)                dgamma = sum_rows dy h,  dbeta = sum_rows dy
//
// Both are bound by memory: 65536 x 1024 bfloat16 values with their checkpoint 60 us forward (338 MB, 5.7 TB/s), 70 to 75 backward (338
// MB, 4.7 TB/s; a plain copy of 4 GB reaches 4.9), and 5 for the join of dgamma and dbeta.  Small ones by the launches: 4096 x 256
// fp32 values 4.4, 5.3 and 2.9 us.  G threads hold a row in registers, P pieces of eight values each (piece i of thread t starts at
// value 8 (t + G i)), so that mean, variance and result need one read; a workgroup walks rows with gains, offsets and, backward,
// the sums of dgamma and dbeta in registers, and requests its next row before it works on the present one.
#include "learner.hpp"
#include "learner_device.hpp"

namespace aq {
namespace {

constexpr int threads_for(int g) { return g <= 64 ? 256 : g; }  // of a workgroup: four wavefronts, or a row
template <int G, int P>
struct RowForm {
    static constexpr int kThreads = threads_for(G);
    static constexpr int kRows = kThreads / G;  // rows at a time in a workgroup
    static_assert(G <= 64 || kRows == 1, "wavefronts of one row share `red`");
    // sum over the threads of a row (G > 64: over LDS; `red` must not be in use by a sum whose barrier some thread has not passed)
    static __device__ __forceinline__ float sum(float s, float* red) {
        s = lanes_sum<G < 64 ? G : 64>(s);
        if constexpr (G > 64) {
            if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
            __syncthreads();
            s = 0.0f;
#pragma unroll
            for (int i = 0; i < G / 64; ++i) s += red[i];
        }
        return s;
    }
};

// a row's values where its checkpoint's 32-value blocks lie: eight codes to a piece, a scale to four threads
struct KeptPiece {
    v2u c;
    uint32_t scale;
    __device__ __forceinline__ void load(const uint8_t* codes, const uint8_t* scales, int64_t row, int64_t blocks, int col, int n) {
        c = v2u{0, 0};
        scale = 127;
        if (n > 0) {
            c = *(const v2u*)(codes + row * blocks * 32 + col);
            scale = scales[row * blocks + (col >> 5)];
        }
    }
    __device__ __forceinline__ void get(float (&v)[8]) const { ckpt8_values(c, ckpt8_step(scale), v); }
};

template <class T, int G, int P, bool KEEP>
__global__ void __launch_bounds__(threads_for(G))
    k_layernorm(const T* __restrict__ x, int64_t ldx, const float* __restrict__ gamma, const float* __restrict__ beta, float eps,
                T* __restrict__ y, int64_t ldy, float* __restrict__ mean_out, float* __restrict__ rstd_out, uint8_t* __restrict__ codes,
                uint8_t* __restrict__ scales, int rows, int cols) {
    using F = RowForm<G, P>;
    __shared__ float red[2][16];
    const int t = threadIdx.x % G;
    const int64_t step = (int64_t)gridDim.x * F::kRows;
    int64_t row = (int64_t)blockIdx.x * F::kRows + threadIdx.x / G;
    if (row >= rows) return;  // (G > 64: the whole workgroup)
    int n[P];
    Piece<float> ga[P], be[P];
    Piece<T> cur[P], next[P];
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const int col = 8 * (t + G * i);
        n[i] = cols - col;
        cur[i].request(x + row * ldx + col, n[i], col);
        ga[i].zero();
        be[i].zero();
        if (gamma) ga[i].load(gamma + col, n[i]);
        if (beta) be[i].load(beta + col, n[i]);
    }
    const int64_t blocks = (cols + 31) / 32;
    for (; row < rows; row += step) {
        if (row + step < rows) {
#pragma unroll
            for (int i = 0; i < P; ++i) next[i].request(x + (row + step) * ldx + 8 * (t + G * i), n[i], 8 * (t + G * i));
        }
        float v[P][8], s = 0.0f;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            if (cols & 7) cur[i].settle(n[i], 8 * (t + G * i));
            cur[i].get(v[i]);
#pragma unroll
            for (int j = 0; j < 8; ++j) s += v[i][j];
        }
        const float mean = F::sum(s, red[0]) / (float)cols;
        float ss = 0.0f;
#pragma unroll
        for (int i = 0; i < P; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float d = j < n[i] ? v[i][j] - mean : 0.0f;
                ss = fmaf(d, d, ss);
            }
        const float rstd = 1.0f / sqrtf(F::sum(ss, red[1]) / (float)cols + eps);
        if (t == 0) {
            if (mean_out) mean_out[row] = mean;
            if (rstd_out) rstd_out[row] = rstd;
        }
#pragma unroll
        for (int i = 0; i < P; ++i) {
            if constexpr (KEEP) {
                const uint32_t scale = ckpt8_scale(most_of4lanes(most_of(cur[i])));
                const int col = 8 * (t + G * i);
                if ((col & ~31) < cols) *(v2u*)(codes + row * blocks * 32 + col) = ckpt8_codes(v[i], scale);
                if ((t & 3) == 0 && col < cols) scales[row * blocks + (col >> 5)] = (uint8_t)scale;
            }
            float o[8], gv[8], bv[8];
            ga[i].get(gv);
            be[i].get(bv);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                o[j] = (v[i][j] - mean) * rstd;
                if (gamma) o[j] *= gv[j];
                if (beta) o[j] += bv[j];
            }
            Piece<T> out;
            out.set(o);
            if (n[i] > 0) out.store(y + row * ldy + 8 * (t + G * i), n[i]);
        }
#pragma unroll
        for (int i = 0; i < P; ++i) cur[i] = next[i];
    }
}

// The gradients.  Every workgroup leaves its sums of dgamma and dbeta in `part` ([workgroup][2][cols]), which k_layernorm_join adds in
// the order of the workgroups; a single workgroup's are the result.
template <class T, bool KEPT, int G, int P>
__global__ void __launch_bounds__(threads_for(G))
    k_layernorm_backward(const T* __restrict__ dy, int64_t lddy, const T* __restrict__ x, int64_t ldx, const uint8_t* __restrict__ codes,
                         const uint8_t* __restrict__ scales, const float* __restrict__ gamma, const float* __restrict__ mean_in,
                         const float* __restrict__ rstd_in, T* __restrict__ dx, int64_t lddx, float* __restrict__ dgamma,
                         float* __restrict__ dbeta, int64_t part_stride, int rows, int cols) {
    using F = RowForm<G, P>;
    using Src = typename std::conditional<KEPT, KeptPiece, Piece<T>>::type;
    // Whether the next row is requested early.  1024 threads have 128 registers each, which would not hold two rows (4096 x 16384: fp32
    // 326 us for 183, bfloat16 150 for 100).
    constexpr bool kAhead = G < 1024;
    __shared__ float red[2][2][16];
    __shared__ float tile[F::kRows > 1 ? F::kRows * 8 * G * P : 1];
    const int t = threadIdx.x % G, grp = threadIdx.x / G;
    const int64_t step = (int64_t)gridDim.x * F::kRows, blocks = (cols + 31) / 32;
    int64_t row = (int64_t)blockIdx.x * F::kRows + grp;
    int n[P];
    float ga[P][8], dg[P][8], db[P][8];
    Piece<T> gy[P], gy_next[P];
    Src in[P], in_next[P];
    float mean = 0.0f, rstd = 0.0f, mean_next = 0.0f, rstd_next = 0.0f;
    auto request = [&](int64_t r, Piece<T>(&g)[P], Src(&s)[P], float& m, float& q) __attribute__((always_inline)) {
        m = mean_in[r];
        q = rstd_in[r];
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const int col = 8 * (t + G * i);
            if constexpr (kAhead) g[i].request(dy + r * lddy + col, n[i], col);
            else g[i].load(dy + r * lddy + col, n[i]);
            if constexpr (KEPT) s[i].load(codes, scales, r, blocks, col, n[i]);
            else if constexpr (kAhead) s[i].request(x + r * ldx + col, n[i], col);
            else s[i].load(x + r * ldx + col, n[i]);
        }
    };
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const int col = 8 * (t + G * i);
        n[i] = cols - col;
        Piece<float> q;
        q.zero();
        if (gamma) q.load(gamma + col, n[i]);
        q.get(ga[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (!gamma) ga[i][j] = 1.0f;
            dg[i][j] = db[i][j] = 0.0f;
        }
    }
    if (kAhead && row < rows) request(row, gy, in, mean, rstd);
    int turn = 0;
    for (; row < rows; row += step) {
        if (!kAhead) request(row, gy, in, mean, rstd);
        else if (row + step < rows) request(row + step, gy_next, in_next, mean_next, rstd_next);
        float g[P][8], h[P][8], s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            if (kAhead && (cols & 7)) {
                gy[i].settle(n[i], 8 * (t + G * i));
                if constexpr (!KEPT) in[i].settle(n[i], 8 * (t + G * i));
            }
            gy[i].get(g[i]);
            in[i].get(h[i]);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                h[i][j] = j < n[i] ? (h[i][j] - mean) * rstd : 0.0f;
                dg[i][j] = fmaf(g[i][j], h[i][j], dg[i][j]);
                db[i][j] += g[i][j];
                g[i][j] *= ga[i][j];
                s1 += g[i][j];
                s2 = fmaf(g[i][j], h[i][j], s2);
            }
        }
        const float c1 = F::sum(s1, red[turn][0]) / (float)cols, c2 = F::sum(s2, red[turn][1]) / (float)cols;
        turn ^= 1;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            float o[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = rstd * (g[i][j] - c1 - h[i][j] * c2);
            Piece<T> out;
            out.set(o);
            if (n[i] > 0) out.store(dx + row * lddx + 8 * (t + G * i), n[i]);
        }
        if constexpr (kAhead) {
#pragma unroll
            for (int i = 0; i < P; ++i) {
                gy[i] = gy_next[i];
                in[i] = in_next[i];
            }
            mean = mean_next;
            rstd = rstd_next;
        }
    }
    // the workgroup's rows join
    auto leave = [&](const float(&v)[P][8], float* out) __attribute__((always_inline)) {
        if (!out) return;
        out += blockIdx.x * part_stride;
        if constexpr (F::kRows > 1) {
            constexpr int kMost = 8 * G * P;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < P; ++i)
#pragma unroll
                for (int j = 0; j < 8; j += 4)
                    *(v4f32*)&tile[grp * kMost + 8 * (t + G * i) + j] = v4f32{v[i][j], v[i][j + 1], v[i][j + 2], v[i][j + 3]};
            __syncthreads();
            for (int c = threadIdx.x; c < cols; c += F::kThreads) {
                float s = 0.0f;
#pragma unroll
                for (int r = 0; r < F::kRows; ++r) s += tile[r * kMost + c];
                out[c] = s;
            }
        } else {
#pragma unroll
            for (int i = 0; i < P; ++i) {
                Piece<float> q;
                q.set(v[i]);
                if (n[i] > 0) q.store(out + 8 * (t + G * i), n[i]);
            }
        }
    };
    leave(dg, dgamma);
    leave(db, dbeta);
}

// sums of the workgroups' parts: 32 columns (of dgamma and dbeta in a row) and 32 slices of the parts to a workgroup
__global__ void __launch_bounds__(1024) k_layernorm_join(const float* __restrict__ part, int parts, int cols, float* __restrict__ dgamma,
                                                         float* __restrict__ dbeta) {
    __shared__ float red[32][33];
    const int c = blockIdx.x * 32 + (threadIdx.x & 31), slice = threadIdx.x >> 5;
    const int64_t width = 2 * (int64_t)cols;
    float s = 0.0f;
    if (c < width)
        for (int i = slice; i < parts; i += 32 * 8) {  // eight on their way at a time
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = i + 32 * j < parts ? part[(i + 32 * j) * width + c] : 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) s += v[j];
        }
    red[slice][threadIdx.x & 31] = s;
    __syncthreads();
    if (slice == 0 && c < width) {
        s = 0.0f;
#pragma unroll
        for (int i = 0; i < 32; ++i) s += red[i][threadIdx.x];
        float* out = c < cols ? dgamma : dbeta;
        if (out) out[c < cols ? c : c - cols] = s;
    }
}

struct Form {
    int g, p;
};
// Threads to a row and pieces a thread, by what the registers hold: the fewest threads that hold it in one piece up to a wavefront, so
// that short rows share one; more than a wavefront from 1025 values on.  4096 x 8192 in {256, 4} / {512, 2}: bfloat16 39.3 / 32.2 us
// forward and 51.2 / 46.8 backward, fp32 63.7 / 58.1 and 94.6 / 89.2.
Form row_form(int64_t cols) {
    if (cols <= 128) return {16, 1};
    if (cols <= 256) return {32, 1};
    if (cols <= 512) return {64, 1};
    if (cols <= 1024) return {64, 2};
    if (cols <= 2048) return {256, 1};
    if (cols <= 4096) return {256, 2};
    if (cols <= 8192) return {512, 2};
    return {1024, 2};
}
template <class Go>
void with_form(const Form& f, Go&& go) {
#define AQ_FORM(GV, PV) \
    if (f.g == GV && f.p == PV) return go(std::integral_constant<int, GV>(), std::integral_constant<int, PV>())
    AQ_FORM(16, 1);
    AQ_FORM(32, 1);
    AQ_FORM(64, 1);
    AQ_FORM(64, 2);
    AQ_FORM(128, 2);
    AQ_FORM(256, 1);
    AQ_FORM(256, 2);
    AQ_FORM(512, 2);
    AQ_FORM(1024, 2);
#undef AQ_FORM
}
int64_t at_a_time(const Form& f) { return threads_for(f.g) / f.g; }

// Workgroups of the backward pass: two turns each until 512 are there; every one leaves 8 bytes a column behind.  65536 x 1024
// bfloat16: with 256 workgroups 99 us, 512 75, 1024 83 and a join twice as long; 512 of 512 threads 75.  4096 x 256 fp32: with one
// workgroup for four turns 7.0 us, for two 5.7.
int64_t backward_workgroups(int64_t rows, int64_t cols) {
    const int64_t turns = (rows + at_a_time(row_form(cols)) - 1) / at_a_time(row_form(cols));
    const int64_t g = (turns + 1) / 2;
    return g < 1 ? 1 : g > 512 ? 512 : g;
}

}  // namespace

aq_status launch_layernorm_forward(const aq_matrix& x, const float* gamma, const float* beta, float eps, const aq_matrix& y,
                                   float* mean, float* rstd, const aq_ckpt8* kept, hipStream_t st) {
    // 16384 x 2048 in {256, 1} / {128, 2}: bfloat16 31.4 / 30.1 us, fp32 61.0 / 59.2; backward, where a workgroup's sums cost more the more
    // there are, fp32 78 / 84
    const Form f = x.cols > 1024 && x.cols <= 2048 ? Form{128, 2} : row_form(x.cols);
    // As many workgroups as run at once; for short rows twice that (65536 x 504 bfloat16 32.9 us / 30.0, but x 1024 58.7 / 60.5)
    const int64_t turns = (x.rows + at_a_time(f) - 1) / at_a_time(f), most = x.cols <= 512 ? 4096 : 2048;
    const unsigned grid = (unsigned)(turns < most ? turns : most);
    return with_dtype(x.dtype, [&](auto t) {
        using T = decltype(t);
        with_form(f, [&](auto g, auto p) {
            using F = RowForm<decltype(g)::value, decltype(p)::value>;
            if (kept)
                k_layernorm<T, decltype(g)::value, decltype(p)::value, true><<<grid, F::kThreads, 0, st>>>(
                    (const T*)x.d, x.ld, gamma, beta, eps, (T*)y.d, y.ld, mean, rstd, (uint8_t*)kept->d_codes, kept->d_scales, (int)x.rows,
                    (int)x.cols);
            else
                k_layernorm<T, decltype(g)::value, decltype(p)::value, false><<<grid, F::kThreads, 0, st>>>(
                    (const T*)x.d, x.ld, gamma, beta, eps, (T*)y.d, y.ld, mean, rstd, nullptr, nullptr, (int)x.rows, (int)x.cols);
        });
        return hip_failed(hipGetLastError()) ? AQ_EHIP : AQ_OK;
    });
}

int64_t layernorm_backward_workspace(int64_t rows, int64_t cols) {
    const int64_t g = backward_workgroups(rows, cols);
    return g > 1 ? g * 2 * cols * (int64_t)sizeof(float) : 0;
}

aq_status launch_layernorm_backward(const aq_matrix& dy, const aq_matrix* x, const aq_ckpt8* kept, const float* gamma, const float* mean,
                                    const float* rstd, const aq_matrix& dx, float* dgamma, float* dbeta, float* ws, hipStream_t st) {
    const int64_t cols = dy.cols, g_wgs = backward_workgroups(dy.rows, cols);
    const Form f = row_form(cols);
    const bool join = g_wgs > 1 && (dgamma || dbeta);
    float* const pg = join ? ws : dgamma;
    float* const pb = join ? ws + cols : dbeta;
    return with_dtype(dy.dtype, [&](auto t) {
        using T = decltype(t);
        with_form(f, [&](auto g, auto p) {
            constexpr int GV = decltype(g)::value, PV = decltype(p)::value;
            using F = RowForm<GV, PV>;
            if (kept)
                k_layernorm_backward<T, true, GV, PV><<<(unsigned)g_wgs, F::kThreads, 0, st>>>(
                    (const T*)dy.d, dy.ld, nullptr, 0, (const uint8_t*)kept->d_codes, kept->d_scales, gamma, mean, rstd, (T*)dx.d, dx.ld, pg, pb,
                    2 * cols, (int)dy.rows, (int)cols);
            else
                k_layernorm_backward<T, false, GV, PV><<<(unsigned)g_wgs, F::kThreads, 0, st>>>(
                    (const T*)dy.d, dy.ld, (const T*)x->d, x->ld, nullptr, nullptr, gamma, mean, rstd, (T*)dx.d, dx.ld, pg, pb, 2 * cols,
                    (int)dy.rows, (int)cols);
        });
        if (hip_failed(hipGetLastError())) return AQ_EHIP;
        if (!join) return AQ_OK;
        k_layernorm_join<<<(unsigned)((2 * cols + 31) / 32), 1024, 0, st>>>(ws, (int)g_wgs, (int)cols, dgamma, dbeta);
        return hip_failed(hipGetLastError()) ? AQ_EHIP : AQ_OK;
    });
}

}  // namespace aq
