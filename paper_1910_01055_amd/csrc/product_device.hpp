// What the tiled products of the learner's operators share.
#pragma once
#include "learner_device.hpp"

namespace aq {

typedef float v16f32 __attribute__((ext_vector_type(16)));

constexpr int kMostLds = 160 * 1024;
// Threads of a workgroup with tiles of S x S: wavefronts two by four, or two by two.
constexpr int tile_threads(int s) { return s == 256 ? 512 : 256; }

// A matrix as a buffer that begins at the rows which a workgroup reads: what lies behind its end comes as zeros, without a branch.
struct Window {
    __amdgpu_buffer_rsrc_t r;
    // of the bytes from `at` (a multiple of 4) on of `size` bytes at `base`
    __device__ __forceinline__ void set(const uint8_t* base, int64_t at, int64_t size) {
        const int64_t left = size - at;
        r = __builtin_amdgcn_make_buffer_rsrc((void*)(base + (left > 0 ? at : 0)), 0, left <= 0 ? 0 : left < kMost ? (int)left : kMost,
                                              0x00020000);
    }
    static constexpr int kMost = 0x7ffffff0, kOutside = (int)0x80000000u;
};
// 16 bytes from `at` bytes behind the window's beginning to LDS, without a register: lane l's go to `to` + 16 l (`to`: the same for the
// whole wavefront).  (A function of its own: inside a template the compiler's host pass drops the kernel without a word.)
__device__ __forceinline__ void load_to_lds(const Window& w, int at, uint8_t* to) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(w.r, (__attribute__((address_space(3))) void*)to, 16, at, 0, 0, 0);
}

// every outstanding LDS operation of the wavefront, then the barrier; loads from memory stay in flight
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// all but the last N of the wavefront's loads from memory are done
template <int N>
__device__ __forceinline__ void wait_loads() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// Which tile and slice a workgroup takes.  Workgroups go to the 8 XCDs, each with an L2 of its own, in turn: every eighth of them
// gets one eighth of all places in a row, and places go along four rows of tiles at once, so that an XCD's workgroups
// read few different rows and columns (weight gradient 65536 x 2048 x 2048, 64 tiles by 4 slices: 545 against 553 us with places in
// order, and half the lines from behind the L2).
struct Place {
    uint32_t m, c, z;
};
__device__ __forceinline__ Place place_of_workgroup(uint32_t gm, uint32_t gc) {
    const uint32_t all = gridDim.x, xcd = blockIdx.x % 8, each = all / 8, more = all % 8;
    const uint32_t p = xcd * each + (xcd < more ? xcd : more) + blockIdx.x / 8;
    const uint32_t z = p / (gm * gc), tile = p % (gm * gc), strip = tile / (4 * gc), in = tile % (4 * gc);
    const uint32_t high = gm - 4 * strip < 4 ? gm - 4 * strip : 4;
    return {4 * strip + in % high, in / high, z};
}

// 32 rows and 32 C columns of sums in the layout of a 32x32 MFMA (lane l: row l mod 32 here, columns 32 i + 8 q + 4 (l / 32) + e),
// rounded and stored as whole lines through 32 kOutRow<T, C> bytes of LDS of the wavefront's own.  get(i, q, e): the sums.  Of the
// rows from `out` on `rows` exist, and `cols` of their columns.
template <class T, int C>
constexpr int kOutRow = 32 * C * (int)sizeof(T) + 16;
template <class T, int C, class Get>
__device__ __forceinline__ void store_rows(uint8_t* place, int lane, T* __restrict__ out, int64_t ld, int64_t rows, int64_t cols, Get&& get) {
    constexpr int kRow = kOutRow<T, C>, kPieces = 32 * C * (int)sizeof(T) / 16, kEach = 16 / (int)sizeof(T);
    uint8_t* const row = place + (lane & 31) * kRow + (lane >> 5) * (4 * (int)sizeof(T));
#pragma unroll
    for (int i = 0; i < C; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float v0 = get(i, q, 0), v1 = get(i, q, 1), v2 = get(i, q, 2), v3 = get(i, q, 3);
            uint8_t* const to = row + (32 * i + 8 * q) * (int)sizeof(T);
            if constexpr (std::is_same<T, float>::value) {
                *(v4f32*)to = v4f32{v0, v1, v2, v3};
            } else {
                typedef T t2 __attribute__((ext_vector_type(2)));
                *(v2u*)to = v2u{__builtin_bit_cast(uint32_t, __builtin_convertvector((v2f32{v0, v1}), t2)),
                                __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f32{v2, v3}), t2))};
            }
        }
#pragma unroll
    for (int k = 0; k < 32 * kPieces / 64; ++k) {
        const int m = (lane + 64 * k) / kPieces, c = (lane + 64 * k) % kPieces * kEach;
        const v4u v = *(const v4u*)(place + m * kRow + c * (int)sizeof(T));
        if (m >= rows) continue;
        T* const to = out + m * ld + c;
        if (c + kEach <= cols) {
            *(v4u_any AQ_GLOBAL*)to = v;
        } else {
            for (int e = 0; e < kEach && c + e < cols; ++e) to[e] = *((const T*)(place + m * kRow) + c + e);
        }
    }
}

}  // namespace aq
