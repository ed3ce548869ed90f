// Operands of attention on the matrix cores, shared by the kernels of equal and of packed sequences: bf16 tiles in LDS that serve both operand forms, and what
// bf16 and float have in common.
#pragma once

#include "device.h"

namespace chimera {

namespace {

typedef bf16_t bf16x8 __attribute__((ext_vector_type(8)));
typedef bf16_t bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int NT = 256, NW = 4, TILE = 32;
constexpr float NEG_BIG = -1.0e30f;
constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f, LN2_LOW = -1.9046543e-9f;     // the float and what it lacks

// ---------------------------------------------------------------------- bf16
__device__ __forceinline__ bf16x8 load_frag(const bf16_t* p, bool ok) {
    bf16x8 z;
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = (bf16_t)0.f;
    return ok ? *reinterpret_cast<const bf16x8*>(p) : z;
}

// LDS tiles: one copy [64 rows][D] per tensor serves BOTH operand forms - a straight
// 16-byte read gives a lane 8 consecutive columns of its row (contraction over columns), the
// transposing read gives it 4 consecutive rows of its column (contraction over rows).  The
// 16-byte chunk c of row r sits at c ^ usw(r); usw is chosen so that both read patterns are
// conflict-free on the 64 banks: a straight read touches 16 consecutive rows at one chunk
// index, a transposing read 4 consecutive rows at 4 consecutive chunks.
template <int D> __device__ __forceinline__ int usw(int r) {
    if (D == 64) { const int h = (r >> 1) & 7; return ((h & 1) << 2) | (h & 2) | (h >> 2); }   // 128-byte rows: bit reversal of r/2
    return ((r & 3) << 2) | ((r >> 2) & 3);                                                     // 256-byte rows
}
template <int D>
__device__ __forceinline__ void dma_utile(const bf16_t* __restrict__ g, int ld, int row0, int row_last, int d, unsigned lds_base,
                                          int wave, int lane) {
    constexpr int KB = 64 * D * 2 / 1024, CPR = D / 8;
#pragma unroll
    for (int n0 = 0; n0 < KB; n0 += NT / WAVE) {
        const int n = n0 + wave;
        const int row = n * (64 / CPR) + lane / CPR;
        const int col = min((lane % CPR) ^ usw<D>(row), d / 8 - 1) << 3;
        lds_dma16(g + (size_t)min(row0 + row, row_last) * ld + col, lds_base + n * 1024);
    }
}
// rows = `row`, contraction step kk over 16 columns
template <int D>
__device__ __forceinline__ bf16x8 frag_us(const bf16_t* tile, int row, int kk, int g) {
    return *reinterpret_cast<const bf16x8*>(tile + row * D + (((kk * 2 + g) ^ usw<D>(row)) << 3));
}
// rows = columns col0 + lane%32 of the tile, contraction over tile rows of 16-step J, in the
// slot order {4g..4g+3, 8+4g..8+4g+3} of a transposed score tile
template <int D>
__device__ __forceinline__ bf16x8 frag_ut(const bf16_t* tile, int col0, int J, int lane) {
    typedef bf16x4 __attribute__((address_space(3))) * lds_v4;
    const int i = lane & 15, g = lane >> 5;
    const int c = (((col0 >> 4) + ((lane >> 4) & 1)) << 1) + ((i >> 1) & 1);
    const int r = 16 * J + 4 * g + (i >> 2);
    const bf16_t* p0 = tile + r * D + ((c ^ usw<D>(r)) << 3) + ((i & 1) << 2);
    const bf16_t* p1 = tile + (r + 8) * D + ((c ^ usw<D>(r + 8)) << 3) + ((i & 1) << 2);
    const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_v4)p0);
    const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_v4)p1);
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

__device__ __forceinline__ bf16x8 pack8(const f32x16& v, int first) {
    bf16x8 o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = (bf16_t)v[first + i];
    return o;
}

// A probability of the backward, exp(score * scale - lse): the difference is rounded once, in natural units, and what the
// product with log2(e) rounds off comes back behind the hardware's exp2.  (From a log-sum-exp in log2 units, rounded on the way
// there, it would carry 1.2 to 1.5 times the error.)
__device__ __forceinline__ float prob(float score, float scale, float lse) {
    const float x = __builtin_fmaf(score, scale, -lse), t = x * LOG2E, e = __builtin_amdgcn_exp2f(t);
    return e == 0.f ? 0.f : __builtin_fmaf(e, __builtin_fmaf(-t, LN2, x), e);        // x may be -inf
}

}  // namespace

}  // namespace chimera
