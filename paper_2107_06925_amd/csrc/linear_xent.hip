// Vocabulary projection and softmax cross-entropy without the logits, forward and backward:
//   z = h W (h [M, H], W stored [H, V]),  lse_t = log sum_v exp z_tv,  loss_t = scale (lse_t - z_t,target)
//   dz_tv = coef_t (exp(z_tv - lse_t) - [v = target_t]),  coef_t = scale dloss_t,  dh = dz W^T,  dW (+)= h^T dz
// A token whose target lies outside [0, V) does not count: loss 0, coef 0, whatever its hidden state holds.
//
// bf16.  The forward's product ends in the statistics of its tile instead of in z: a (maximum, sum) pair per row and tile,
// which a second kernel combines.  The backward forms z again, a piece of the vocabulary at a time, and ends in dz of
// that piece; two products take it from there.  One launch per piece holds both, and z of the next piece, so that no product's last round leaves
// the chip idle.
// dz is kept as two fp16 numbers, hi + lo.  dW takes both, because it is a float sum: one bf16 dz would leave it 2e-3 off, two 3e-6, two of fp16
// (11 bits each) 1e-7.  dh is rounded to bf16 itself, and takes hi: a bf16 dz would add as much error as that rounding.  fp16's range is met by powers of two:
//   dz_t times 2^lift_t: the row's coef comes to lie in [2^13, 2^14);
//   W's rows within a piece times 2^raise_i: the row's largest number in [2^14, 2^15), where fp16 holds a bf16 number exactly down to 2^-28 of it;
//   h_t times 2^(shift - lift_t), for dW, which sums over tokens: one shift for all, the largest that keeps all rows below 2^15.
// The products' epilogues take the powers off again.
//
// float.  The framework's float products on pieces that are in memory, z's ending in dz in the backward.
#include "gemm_tiles.h"
#include "spans.h"

#include <array>
#include <climits>
#include <cmath>
#include <cstdlib>
#include <initializer_list>
#include <utility>

namespace chimera {
namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LOWEST = -3.0e38f;              // stands for the maximum of nothing: differences from it stay finite
constexpr int TOKEN_PAD = 32;                   // the weight gradient's contraction, two rows a token, is walked in steps of 64
constexpr int ROW_THREADS = 256, ROW_FLY = 4;   // float rows: loads in flight a thread

// f over the four lanes that hold a row of a 16x16 tile (l, l ^ 16, l ^ 32, l ^ 48)
template <typename F> __device__ __forceinline__ float fold_row(float v, F f) {
    v = fold32(v, f);
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return f(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float add_f(float a, float b) { return a + b; }
__device__ __forceinline__ bool counts(int target, int vocab) { return (unsigned)target < (unsigned)vocab; }

// (maximum, sum of exp(z - maximum)) of a and b together
__device__ __forceinline__ float2 join(float2 a, float2 b) {
    const float m = fmaxf(a.x, b.x);
    return make_float2(m, a.y * __builtin_amdgcn_exp2f((a.x - m) * LOG2E) + b.y * __builtin_amdgcn_exp2f((b.x - m) * LOG2E));
}

// ---- what the forward's tiles end in.  A lane holds runs of four columns of the rows l%16 of its 16x16 tiles (Acc16), so a row's statistics over
// a wavefront's 64 columns are 16 numbers and a fold over four lanes; the wavefronts of a tile row join theirs in LDS.
template <int BM, int BN> struct StatsEnd {
    const int* targets;
    float2* stats;               // [tile column][token], from this launch's first on
    float* at_target;            // [token]
    int m, vocab;
    __device__ __forceinline__ void begin(int, int) {}
    template <int TO, int TN2, typename Acc>
    __device__ __forceinline__ void end(const Acc& out, char* lds, int i0, int rb0, int cb0, int tile_n, int, int lane) const {
        constexpr int PARTS = BN / 64;
        static_assert(TN2 == 2, "wavefronts of 64 columns");
        float2 (*tab)[BM] = reinterpret_cast<float2 (*)[BM]>(lds);
        const int l16 = lane & 15, g = lane >> 4, part = cb0 / 64 % PARTS;
        const bool whole = cb0 + 64 <= vocab;
#pragma unroll
        for (int a = 0; a < 2 * TO; ++a) {
            const int row = rb0 + a * 16 + l16;
            float v[16];
#pragma unroll
            for (int b = 0; b < 4; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[4 * b + e] = out.acc[a][b][e];
                    if (!whole && cb0 + b * 16 + 4 * g + e >= vocab) v[4 * b + e] = -INFINITY;
                }
            float top = LOWEST;
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, v[i]);
            top = fold_row(top, [](float x, float y) { return fmaxf(x, y); });
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) sum += __builtin_amdgcn_exp2f((v[i] - top) * LOG2E);
            sum = fold_row(sum, add_f);
            if (g == 0) tab[part][row - i0] = make_float2(top, sum);
            const int at = row < m ? targets[row] - cb0 : -1;              // (a column of this wavefront: at most one lane of the row's four holds it)
            if (__any((unsigned)at < 64u)) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (at == (i >> 2) * 16 + 4 * g + (i & 3) && at + cb0 < vocab) at_target[row] = v[i];
            }
        }
        __syncthreads();
        const int tid = threadIdx.x;
        if (tid < BM && i0 + tid < m) {
            float2 s = tab[0][tid];
#pragma unroll
            for (int p = 1; p < PARTS; ++p) s = join(s, tab[p][tid]);
            stats[(size_t)tile_n * m + i0 + tid] = s;
        }
    }
};

// Columns [0, wide) on 256x256 tiles, a whole number of rounds of them, and what is left on 128x128 tiles, begun first: a last round of a few large tiles
// costs as much as a full one.  Matrix instructions bound it: 2048 x 1600 x 50257 266 to 270 us, 1.22 PFLOP/s, a large square product of this library's 1.4 to 1.5.
struct StatsPass {
    const bf16_t *h, *w;
    const int* targets;
    float2* stats;
    float* at_target;
    int m, vocab, k, ldh, ldw, wide;
    int small;                   // workgroups of 128x128 tiles
    struct Raster { int tiles_m, tiles_n, group_m, band; } r256, r128;
};
__global__ __launch_bounds__(512, 2) void xent_stats_kernel(StatsPass p) {
    __shared__ __attribute__((aligned(1024))) char lds[RingLds<256, 256, 2, 4, 1>::BYTES];
    static_assert(sizeof lds >= RingLds<128, 128, 2, 2, 2>::BYTES, "the larger of the two");
    const int n = (p.vocab + 7) & ~7, id = blockIdx.x;
    if (id < p.small)
        gemm_ring_tile<128, 128, 2, 2, 2, true, false, EPI_OWN>(lds, p.h, p.w, nullptr, nullptr, nullptr, nullptr, p.m, n, p.k, p.ldh, p.ldw, EPI_OWN, 0, 0, p.r128.tiles_m,
                                                                p.r128.tiles_n, p.r128.group_m, id, nullptr, true, p.wide, Ahead{nullptr, 0}, p.r128.band,
                                                                StatsEnd<128, 128>{p.targets, p.stats + (size_t)(p.wide / 256) * p.m, p.at_target, p.m, p.vocab});
    else
        gemm_ring_tile<256, 256, 2, 4, 1, true, false, EPI_OWN, false, false, true>(lds, p.h, p.w, nullptr, nullptr, nullptr, nullptr, p.m, n, p.k, p.ldh, p.ldw, EPI_OWN, 0,
                                                                                    0, p.r256.tiles_m, p.r256.tiles_n, p.r256.group_m, id - p.small, nullptr, true, 0,
                                                                                    Ahead{nullptr, 0}, p.r256.band,
                                                                                    StatsEnd<256, 256>{p.targets, p.stats, p.at_target, p.m, p.vocab});
}

// The pairs of a row, joined by 16 lanes, which take every sixteenth pair and join theirs in order; then the loss.  Up to JOIN_ALONE tokens one
// workgroup of 64 rows at a time does it all, beyond, workgroups of 16 rows leave the sum to a launch of its own (fixed order either way).
constexpr int JOIN_ALONE = 256;
template <int ROWS>
__global__ __launch_bounds__(16 * ROWS) void xent_join_kernel(const float2* __restrict__ stats, const float* __restrict__ at_target, const int* __restrict__ targets,
                                                              int m, int vocab, int parts, float scale, float* __restrict__ loss_rows, float* __restrict__ lse,
                                                              float* __restrict__ loss) {
    __shared__ float2 tab[16][ROWS];
    const int r = threadIdx.x % ROWS, q = threadIdx.x / ROWS;
    float sum = 0.f;
    for (int r0 = blockIdx.x * ROWS; r0 < m; r0 += gridDim.x * ROWS) {
        const int row = r0 + r;
        float2 s = make_float2(LOWEST, 0.f);
        if (row < m) {
            int p = q;
            for (; p + 48 < parts; p += 64) {
                float2 u[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) u[i] = stats[(size_t)(p + 16 * i) * m + row];
#pragma unroll
                for (int i = 0; i < 4; ++i) s = join(s, u[i]);
            }
            for (; p < parts; p += 16) s = join(s, stats[(size_t)p * m + row]);
        }
        tab[q][r] = s;
        __syncthreads();
        if (!q && row < m) {
#pragma unroll
            for (int i = 1; i < 16; ++i) s = join(s, tab[i][r]);
            const float l = s.x + logf(s.y), own = counts(targets[row], vocab) ? scale * (l - at_target[row]) : 0.f;
            lse[row] = l;
            loss_rows[row] = own;
            sum += own;
        }
        __syncthreads();
    }
    if constexpr (ROWS == WAVE) {                // (the first wavefront holds the rows' sums)
        if (!loss || q) return;
        sum = wave_sum(sum);
        if (threadIdx.x == 0) loss[0] += sum;
    }
}

// ---- backward
// A token's coef, and the power of two that brings it to [2^13, 2^14) (0 where it is zero)
__device__ __forceinline__ float coef_of(const int* targets, const float* dloss, float scale, int t, int m, int vocab) {
    return t < m && counts(targets[min(t, m - 1)], vocab) ? (dloss ? scale * dloss[min(t, m - 1)] : scale) : 0.f;
}
__device__ __forceinline__ int lift_of(float coef) { return coef != 0.f ? 14 - __builtin_amdgcn_frexp_expf(coef) : 0; }      // coef = f 2^exp, f in [1/2, 1)

// The largest shift that each token allows: h_t 2^(shift - lift_t) stays below 2^15.  INT_MAX: any.  One wavefront per token.
__global__ __launch_bounds__(ROW_THREADS) void xent_room_kernel(const bf16_t* __restrict__ h, int ldh, const int* __restrict__ targets, const float* __restrict__ dloss,
                                                                float scale, int m, int cols, int vocab, int* __restrict__ room) {
    const int t = blockIdx.x * (ROW_THREADS / WAVE) + threadIdx.x / WAVE, lane = threadIdx.x % WAVE;
    if (t >= m) return;
    const float coef = coef_of(targets, dloss, scale, t, m, vocab);
    float top = 0.f;
    if (coef != 0.f)
        for (int c = lane; c < cols / 8; c += WAVE) {
            float x[8];
            load_vec<bf16_t>(h + (size_t)t * ldh + c * 8, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[e]));
        }
    top = wave_max(top);
    if (lane == 0) room[t] = top > 0.f ? 15 - __builtin_amdgcn_frexp_expf(top) + lift_of(coef) : INT_MAX;
}

// What the launches of a pass work on
struct Piece {
    int v0, cols, ld;                // first column of the vocabulary, columns, columns rounded up to 8
    _Float16* dz;                    // [mp][2][ld]: hi and lo of a token
    _Float16* w;                     // [hidden, ldp] W's rows, times 2^raise
    int* raise;                      // [hidden]
    float* dw;                       // [parts][hidden, ld], where dW's contraction is cut
};
struct Pass {
    const bf16_t *h, *w;
    const int* targets;
    const float *lse, *dloss;
    float scale;
    int m, mp, hidden, vocab, ldh, ldw, ldp;
    int *room, *shift;
    _Float16* rows;                  // [hidden, mp]: h_t 2^(shift - lift_t), transposed
    Piece now, next;                 // the products' piece, and the one that dz is formed of
    Piece past;                      // whose parts of dW are added
    // dW: columns of `now`
    float* dw;
    int lddw, dw_flags, dw_per, dw_splits;       // tokens a part
    // dh: float slabs [split][m, hidden]
    float* slabs;
    int k_per, dh_flags;
    int w_rows;                      // rows of W a workgroup
    int first[6], count[6];          // workgroups of each kind: dW, dh, dz, W's rows, h^T, sums of dW; and the rasters of their tiles
    struct Raster { int tiles_m, tiles_n, group_m, band; } dw_r, dh_r, dz_r;
};

// dW (+)= h^T dz, 2^shift taken off
struct ColumnsEnd {
    float* c;
    const int* shift;
    int m, n, ldc, flags, pair;
    __device__ __forceinline__ void begin(int, int) {}
    template <int TO, int TN2, typename Acc>
    __device__ __forceinline__ void end(const Acc& out, char* lds, int, int rb0, int cb0, int, int wave, int lane) const {
        float* slab = reinterpret_cast<float*>(lds) + (size_t)wave * EpiSlab<TN2>::FLOATS;
        accumulate<false, true, TO, TN2>(out, slab, rb0, cb0, m, n, ldc, *shift, c, flags, lane);
    }
};
// a split of dh, of the columns' 2^raise alone: the tokens' 2^lift goes when the slabs are added
struct SlabEnd {
    float* c;
    const int* raise;
    int m, n, flags;
    __device__ __forceinline__ void begin(int, int) {}
    template <int TO, int TN2, typename Acc>
    __device__ __forceinline__ void end(const Acc& out, char* lds, int, int rb0, int cb0, int, int wave, int lane) const {
        constexpr int CPR = EpiSlab<TN2>::WN / 4, RPP = 64 / CPR, NP = 32 / RPP;
        float* slab = reinterpret_cast<float*>(lds) + (size_t)wave * EpiSlab<TN2>::FLOATS;
        const int pr = lane / CPR, piece = lane % CPR, gcol = cb0 + piece * 4, lcol = min(gcol, n - 4);
        const bool reads = !(flags & ACCUM_OVERWRITE);
        const int4 r = *reinterpret_cast<const int4*>(raise + lcol);
        static_for<TO>([&](auto a_c) {
            constexpr int a = decltype(a_c)::value;
            f32x4 old[NP];
            if (reads)
#pragma unroll
                for (int j = 0; j < NP; ++j)
                    old[j] = *reinterpret_cast<const f32x4*>(c + (size_t)min(rb0 + a * 32 + j * RPP + pr, m - 1) * n + lcol);
            out.template put<a>(slab, lane);
            __builtin_amdgcn_s_waitcnt(0xc07f);                   // lgkmcnt(0): the slab is written (wavefront-private)
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int j = 0; j < NP; ++j) {
                const int lr = j * RPP + pr, row = rb0 + a * 32 + lr;
                f32x4 v = *reinterpret_cast<const f32x4*>(EpiSlab<TN2>::at(slab, lr, piece));
                v = f32x4{ldexpf(v[0], -r.x), ldexpf(v[1], -r.y), ldexpf(v[2], -r.z), ldexpf(v[3], -r.w)};
                if (reads) v += old[j];
                if (row < m && gcol < n) *reinterpret_cast<f32x4*>(c + (size_t)row * n + gcol) = v;
            }
            __builtin_amdgcn_wave_barrier();                      // all lanes have read the slab before it is rewritten
        });
    }
};
// dz of a piece.  Behind a tile's k loop come 256 KB of stores, 65536 exponentials and conversions, with the matrix pipes idle: of a round of 256 tiles at hidden
// 2048, 61 us, some 20 (the stores 6, the exponentials 3).  A band of 32 rows looks for targets only where it holds one.
struct RowInfo { float lse, scaled; int at; };              // coef 2^lift (0: the token does not count), the target's column in the piece
template <int BM> struct GradEnd {
    const Pass* p;
    float lse, weight;
    int target;
    __device__ __forceinline__ void begin(int i0, int tid) {                     // requests only: their values are looked at behind the k loop
        const int t = min(i0 + tid, p->m - 1);
        lse = p->lse[t];
        target = p->targets[t];
        weight = 1.0f;
        if (p->dloss) weight = p->dloss[t];
    }
    template <int TO, int TN2, typename Acc>
    __device__ __forceinline__ void end(const Acc& out, char* lds, int i0, int rb0, int cb0, int, int wave, int lane) const {
        constexpr int CPR = EpiSlab<TN2>::WN / 8, RPP = 64 / CPR, NP = 32 / RPP;
        RowInfo* tab = reinterpret_cast<RowInfo*>(lds + 8 * EpiSlab<TN2>::FLOATS * sizeof(float));
        float* slab = reinterpret_cast<float*>(lds) + (size_t)wave * EpiSlab<TN2>::FLOATS;
        const int tid = threadIdx.x, cols = p->next.cols, ld = p->next.ld, mp = p->mp;
        if (tid < BM) {
            const float coef = i0 + tid < p->m && counts(target, p->vocab) ? p->scale * weight : 0.f;
            tab[tid] = {lse, ldexpf(coef, lift_of(coef)), coef != 0.f ? target - p->next.v0 : -1};
        }
        __syncthreads();
        const int pr = lane / CPR, pc = lane % CPR * 8, col = cb0 + pc;
        _Float16* const first = p->next.dz + (size_t)(rb0 + pr) * 2 * ld + col;
        static_for<TO>([&](auto a_c) {
            constexpr int a = decltype(a_c)::value;
            if (rb0 + a * 32 >= mp) return;                       // (mp is a multiple of 32)
            out.template put<a>(slab, lane);
            const bool usual = cb0 + EpiSlab<TN2>::WN <= cols && !__any((unsigned)(tab[rb0 - i0 + a * 32 + (lane & 31)].at - cb0) < (unsigned)EpiSlab<TN2>::WN);
            __builtin_amdgcn_s_waitcnt(0xc07f);                   // lgkmcnt(0): the slab is written (wavefront-private)
            __builtin_amdgcn_wave_barrier();
            auto rows = [&](auto usual_c) {
#pragma unroll
                for (int j = 0; j < NP; ++j) {
                    const int lr = a * 32 + j * RPP + pr;
                    const RowInfo r = tab[rb0 - i0 + lr];
                    float v[8];
                    load_vec<float>(EpiSlab<TN2>::at(slab, j * RPP + pr, pc / 4), v);
                    load_vec<float>(EpiSlab<TN2>::at(slab, j * RPP + pr, pc / 4 + 1), v + 4);
                    typedef float f32x2 __attribute__((ext_vector_type(2)));
                    typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
                    f16x2 hi[4], lo[4];
#pragma unroll
                    for (int e = 0; e < 8; e += 2) {
                        f32x2 d;
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            // (the smaller of 126 and what is no number is 126: a token that does not count has zeros)
                            float x = __builtin_amdgcn_exp2f(fminf((v[e + q] - r.lse) * LOG2E, 126.0f));
                            if constexpr (!decltype(usual_c)::value) {
                                x -= col + e + q == r.at ? 1.0f : 0.0f;
                                if (col + e + q >= cols) x = 0.f;
                            }
                            d[q] = r.scaled * x;
                        }
                        hi[e / 2] = __builtin_convertvector(d, f16x2);
                        const f32x2 rest = d - __builtin_convertvector(hi[e / 2], f32x2);
                        lo[e / 2] = __builtin_convertvector(rest, f16x2);
                    }
                    if constexpr (!decltype(usual_c)::value)
                        if (col >= ld) continue;
                    _Float16* to = first + (size_t)(a * 32 + j * RPP) * (2 * ld);
                    *reinterpret_cast<uint4*>(to) = *reinterpret_cast<const uint4*>(hi);
                    *reinterpret_cast<uint4*>(to + ld) = *reinterpret_cast<const uint4*>(lo);
                }
            };
            if (usual) rows(std::true_type{});
            else rows(std::false_type{});
            __builtin_amdgcn_wave_barrier();                      // all lanes have read the slab before it is rewritten
        });
    }
};

// A row of W within the next piece as fp16 numbers times 2^raise; columns behind the vocabulary as zeros, whatever they hold.  Looked over
// once, and once more, out of the cache, to be written.  A workgroup takes w_rows of them, 8 / w_rows wavefronts each.
__device__ __forceinline__ void raise_rows(const Pass& p, int id, char* lds) {
    const int waves = 8 / p.w_rows, wave = threadIdx.x / WAVE, at = wave % waves * WAVE + threadIdx.x % WAVE, ld = p.next.ld, cols = p.next.cols;
    const int own = id * p.w_rows + wave / waves, i = min(own, p.hidden - 1);
    const bf16_t* src = p.w + (size_t)i * p.ldw + p.next.v0;
    _Float16* to = p.next.w + (size_t)i * p.ldp;
    float* part = reinterpret_cast<float*>(lds);
    constexpr int FLY = 8;
    const int STRIDE = waves * WAVE * 8;
    float top = 0.f;
    auto look = [&](int c, const uint4& q) {
        float x[8];
        load_vec<bf16_t>(reinterpret_cast<const bf16_t*>(&q), x);
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, c + e < cols ? fabsf(x[e]) : 0.f);
    };
    for (int c0 = at * 8; c0 < ld; c0 += FLY * STRIDE) {
        uint4 q[FLY];
#pragma unroll
        for (int u = 0; u < FLY; ++u) q[u] = *reinterpret_cast<const uint4*>(src + min(c0 + u * STRIDE, ld - 8));      // (what is behind the row counts once more)
#pragma unroll
        for (int u = 0; u < FLY; ++u) look(min(c0 + u * STRIDE, ld - 8), q[u]);
    }
    top = wave_max(top);
    if (threadIdx.x % WAVE == 0) part[wave] = top;
    __syncthreads();
    for (int k = 0; k < waves; ++k) top = fmaxf(top, part[wave / waves * waves + k]);
    if (own >= p.hidden) return;
    const int up = top > 0.f ? 15 - __builtin_amdgcn_frexp_expf(top) : 0;
    if (at == 0) p.next.raise[i] = up;
    for (int c0 = at * 8; c0 < ld; c0 += FLY * STRIDE) {
        uint4 q[FLY];
#pragma unroll
        for (int u = 0; u < FLY; ++u) q[u] = *reinterpret_cast<const uint4*>(src + min(c0 + u * STRIDE, ld - 8));
#pragma unroll
        for (int u = 0; u < FLY; ++u) {
            const int c = c0 + u * STRIDE;
            float x[8];
            load_vec<bf16_t>(reinterpret_cast<const bf16_t*>(&q[u]), x);
            f16x8 y;
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = c + e < cols ? (_Float16)ldexpf(x[e], up) : (_Float16)0.f;
            if (c < ld) *reinterpret_cast<f16x8*>(to + c) = y;
        }
    }
}
// h^T times 2^(shift - lift); tokens that do not count, and the padding behind the last one, as zeros: their dz is zero, but h may hold anything.
// Transposed, so that dW's A is contiguous along the contraction: a tile then asks for its 32 tokens of a step once for both parts of dz (dW of 8192 x 2048 x 65536
// 6867 -> 6822 us in all, 6813 -> 6714 with half of the requests), and its lines can be touched ahead (a step of dW 3080 -> 2457 clocks).
constexpr int TURN_TOKENS = 64, TURN_COLS = 256, TURN_WGS = 1024;
__device__ __forceinline__ void turn_rows(const Pass& p, int id, int wgs, char* lds) {
    int* part = reinterpret_cast<int*>(lds);
    constexpr int LD = TURN_TOKENS + 8;
    _Float16* tile = reinterpret_cast<_Float16*>(lds + 64);        // [64 columns][LD]
    int least = INT_MAX;
    for (int t = threadIdx.x; t < p.m; t += 512) least = min(least, p.room[t]);
#pragma unroll
    for (int o = 32; o; o >>= 1) least = min(least, __shfl_xor(least, o, WAVE));
    if (threadIdx.x % WAVE == 0) part[threadIdx.x / WAVE] = least;
    __syncthreads();
    for (int i = 0; i < 8; ++i) least = min(least, part[i]);
    const int shift = least == INT_MAX ? 0 : least;
    if (id == 0 && threadIdx.x == 0) *p.shift = shift;
    const int groups = (p.hidden + TURN_COLS - 1) / TURN_COLS, units = (p.mp + TURN_TOKENS - 1) / TURN_TOKENS * groups;
    const int a = threadIdx.x >> 3, b = threadIdx.x & 7;          // token and 8 columns on the way in, column and 8 tokens on the way out
    for (int u = id; u < units; u += wgs) {
        const int t0 = u / groups * TURN_TOKENS, g0 = u % groups * TURN_COLS;
        const float coef = coef_of(p.targets, p.dloss, p.scale, t0 + a, p.m, p.vocab);
        const int up = shift - lift_of(coef);
        for (int c0 = g0; c0 < min(g0 + TURN_COLS, p.hidden); c0 += 64) {
            if (c0 + b * 8 < p.hidden) {
                float x[8];
                load_vec<bf16_t>(p.h + (size_t)min(t0 + a, p.m - 1) * p.ldh + c0 + b * 8, x);
#pragma unroll
                for (int e = 0; e < 8; ++e) tile[(b * 8 + e) * LD + a] = coef != 0.f ? (_Float16)ldexpf(x[e], up) : (_Float16)0.f;
            }
            __syncthreads();
            if (c0 + a < p.hidden && t0 + b * 8 < p.mp)
                *reinterpret_cast<f16x8*>(p.rows + (size_t)(c0 + a) * p.mp + t0 + b * 8) = *reinterpret_cast<const f16x8*>(tile + a * LD + b * 8);
            __syncthreads();
        }
    }
}

// dW (+)= the parts of a piece
constexpr int SUM_WGS = 512;
__device__ __forceinline__ void sum_columns(const Pass& p, int id, int wgs) {
    const int fours = p.past.ld / 4;
    const size_t stride = (size_t)p.hidden * p.past.ld, units = (size_t)p.hidden * fours;
    for (size_t u = (size_t)id * 512 + threadIdx.x; u < units; u += (size_t)wgs * 512) {
        const int i = (int)(u / fours), c = (int)(u % fours) * 4;
        const float* from = p.past.dw + (size_t)i * p.past.ld + c;
        float* to = p.dw + (size_t)i * p.lddw + p.past.v0 + c;
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
        const bool whole = c + 4 <= p.past.cols;
        if (whole && !(p.dw_flags & ACCUM_OVERWRITE)) v = *reinterpret_cast<const f32x4*>(to);
        for (int k = 0; k < p.dw_splits; ++k) v += *reinterpret_cast<const f32x4*>(from + k * stride);
        if (whole) *reinterpret_cast<f32x4*>(to) = v;
        else
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (c + e < p.past.cols) to[e] = p.dw_flags & ACCUM_OVERWRITE ? v[e] : to[e] + v[e];
    }
}

// One launch: dW and dh of a piece, dz and the rows of W of the next, the sums of dW's parts of the one before, and, in the first, h^T.  Tiles of DW x DW for
// dW, of TOK x TOK for the products over tokens.  Four products (z, dh, dW of either part of dz), a third more
// than a dz in one part needs: 8192 x 2048 x 65536 6.36 to 6.47 ms, 1.36 to 1.38 PFLOP/s, where the chip's power is what bounds it (a step of dW takes 2457 clocks for 2048 of matrix instructions, at
// about 1.7 GHz); 2048 x 1600 x 50257 1.29 to 1.31 ms, 1.0: tiles of 25 to 64 steps, each with some 20 us of first loads and stores on a CU that holds no other.
template <int DW, int TOK>
__global__ __launch_bounds__(512, 2) void xent_pass_kernel(Pass p) {
    constexpr int BYTES = RingLds<256, 256, 2, 4, 1>::BYTES;
    static_assert(RingLds<128, 128, 2, 2, 2>::BYTES <= BYTES, "the larger of the two");
    static_assert(BYTES >= 8 * EpiSlab<2>::FLOATS * sizeof(float) + 256 * sizeof(RowInfo), "room for the slabs and the rows");
    __shared__ __attribute__((aligned(1024))) char lds[BYTES];
    const int block = blockIdx.x;
#define XENT_TILE(T, AKC, BKC, F16, PAIRED, A, B, M, N, K, LDA, LDB, R, ID, BAND, XCD, END)                                                                          \
    do {                                                                                                                                                       \
        if constexpr (T == 256)                                                                                                                                \
            gemm_ring_tile<256, 256, 2, 4, 1, AKC, BKC, EPI_OWN, F16, PAIRED, true>(lds, A, B, nullptr, nullptr, nullptr, nullptr, M, N, K, LDA, LDB, EPI_OWN, 0, 0,  \
                                                                              R.tiles_m, R.tiles_n, R.group_m, ID, nullptr, XCD, 0, Ahead{nullptr, 0}, BAND, END); \
        else                                                                                                                                                   \
            gemm_ring_tile<128, 128, 2, 2, 2, AKC, BKC, EPI_OWN, F16, PAIRED>(lds, A, B, nullptr, nullptr, nullptr, nullptr, M, N, K, LDA, LDB, EPI_OWN, 0, 0,  \
                                                                              R.tiles_m, R.tiles_n, R.group_m, ID, nullptr, XCD, 0, Ahead{nullptr, 0}, BAND, END); \
    } while (0)
    auto kind = [&](int k) { return (unsigned)(block - p.first[k]) < (unsigned)p.count[k]; };
    if (kind(0)) {
        const int tiles = p.dw_r.tiles_m * p.dw_r.tiles_n, at = block - p.first[0], part = __builtin_amdgcn_readfirstlane(at / tiles), t0 = part * p.dw_per;
        const bool cut = p.dw_splits > 1;
        const ColumnsEnd end{cut ? p.now.dw + (size_t)part * p.hidden * p.now.ld : p.dw + p.now.v0, p.shift, p.hidden, cut ? p.now.ld : p.now.cols,
                             cut ? p.now.ld : p.lddw, cut ? ACCUM_OVERWRITE : p.dw_flags, p.now.ld};
        XENT_TILE(DW, true, false, true, true, (const bf16_t*)p.rows + t0, (const bf16_t*)p.now.dz + (size_t)t0 * 2 * p.now.ld, p.hidden, p.now.ld,
                  2 * min(p.dw_per, p.mp - t0), p.mp, 2 * p.now.ld, p.dw_r, at - part * tiles, p.dw_r.band, true, end);
    } else if (kind(1)) {
        const int at = block - p.first[1], tiles = p.dh_r.tiles_m * p.dh_r.tiles_n, total = p.count[1];
        const int xcd = at & 7, local = at >> 3, pid = xcd * (total >> 3) + min(xcd, total & 7) + local;
        const int split = __builtin_amdgcn_readfirstlane(pid / tiles), k0 = split * p.k_per;
        const SlabEnd end{p.slabs + (size_t)split * p.m * p.hidden, p.now.raise, p.m, p.hidden, p.dh_flags};
        XENT_TILE(TOK, true, true, true, false, (const bf16_t*)p.now.dz + k0, (const bf16_t*)p.now.w + k0, p.m, p.hidden, min(p.k_per, p.now.ld - k0), 2 * p.now.ld,
                  p.ldp, p.dh_r, pid - split * tiles, 0, false, end);
    } else if (kind(2)) {
        XENT_TILE(TOK, true, false, false, false, p.h, p.w + p.next.v0, p.m, p.next.ld, p.hidden, p.ldh, p.ldw, p.dz_r, block - p.first[2], p.dz_r.band, true,
                  (GradEnd<TOK>{&p, 0.f, 0.f, 0}));
    } else if (kind(3)) {
        raise_rows(p, block - p.first[3], lds);
    } else if (kind(4)) {
        turn_rows(p, block - p.first[4], p.count[4], lds);
    } else {
        sum_columns(p, block - p.first[5], p.count[5]);
    }
#undef XENT_TILE
}

// dh = the slabs' sum, the tokens' 2^lift taken off (bf16); float: with the product of the last vocabulary columns, fewer than 8, that no slab holds
// (what lies beside them in W's rows does not count and need not be a number).  A thread owns 4 columns of a token.  Bound by the slabs: 2048 x 1600 in
// three 10 us.
template <typename T>
__global__ __launch_bounds__(ROW_THREADS) void xent_dh_sum_kernel(const float* __restrict__ slabs, int splits, const T* __restrict__ dz, int ldz,
                                                                  const T* __restrict__ w, int ldw, int tail, const int* __restrict__ targets,
                                                                  const float* __restrict__ dloss, float scale, int vocab, int m, int n, T* __restrict__ dh, int lddh) {
    for (size_t at = (size_t)blockIdx.x * ROW_THREADS + threadIdx.x; at < (size_t)m * (n / 4); at += (size_t)gridDim.x * ROW_THREADS) {
        const int t = (int)(at / (n / 4)), c = (int)(at % (n / 4)) * 4;
        const float* from = slabs + (size_t)t * n + c;
        const size_t stride = (size_t)m * n;
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
        int s = 0;
        for (; s + 4 <= splits; s += 4) {
            f32x4 u[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) u[i] = *reinterpret_cast<const f32x4*>(from + (s + i) * stride);
#pragma unroll
            for (int i = 0; i < 4; ++i) v += u[i];
        }
        for (; s < splits; ++s) v += *reinterpret_cast<const f32x4*>(from + s * stride);
        T* to = dh + (size_t)t * lddh + c;
        if constexpr (sizeof(T) == 4) {
            for (int j = 0; j < tail; ++j) {
                const float d = dz[(size_t)t * ldz + j];
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] += d * w[(size_t)(c + i) * ldw + j];
            }
            *reinterpret_cast<f32x4*>(to) = v;
        } else {
            const int lift = lift_of(coef_of(targets, dloss, scale, t, m, vocab));
            *reinterpret_cast<bf16x4*>(to) = bf16x4{(bf16_t)ldexpf(v[0], -lift), (bf16_t)ldexpf(v[1], -lift), (bf16_t)ldexpf(v[2], -lift), (bf16_t)ldexpf(v[3], -lift)};
        }
    }
}

// float: what a piece's product needs to know of a token, and the rows of h that the weight gradient takes (may be null), tokens that do not count as zeros
__global__ __launch_bounds__(ROW_THREADS) void xent_rows_f32_kernel(const float* __restrict__ h, int ldh, const int* __restrict__ targets, const float* __restrict__ lse,
                                                                    const float* __restrict__ dloss, float scale, int m, int cols, int vocab, XentRow* __restrict__ info,
                                                                    float* __restrict__ out) {
    const int t = blockIdx.x * (ROW_THREADS / WAVE) + threadIdx.x / WAVE, lane = threadIdx.x % WAVE;
    if (t >= m) return;
    const float coef = coef_of(targets, dloss, scale, t, m, vocab);
    if (lane == 0) info[t] = {lse[t], coef, targets[t], vocab};
    if (!out) return;
    for (int c = lane * 4; c < cols; c += WAVE * 4) {
        float x[4];
        load_vec<float>(h + (size_t)t * ldh + c, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = coef != 0.f ? x[e] : 0.f;
        store_vec<float>(out + (size_t)t * cols + c, x);
    }
}

// ---- float: a piece of z is in memory, [m, ld], of which `cols` columns from v0 on count
__global__ __launch_bounds__(ROW_THREADS) void xent_stats_f32_kernel(const float* __restrict__ z, int ld, int cols, int v0, int vocab, const int* __restrict__ targets,
                                                                     float2* __restrict__ stats, float* __restrict__ at_target) {
    __shared__ float2 part[ROW_THREADS / WAVE];
    const int t = blockIdx.x, tid = threadIdx.x;
    const float* row = z + (size_t)t * ld;
    float2 s = make_float2(LOWEST, 0.f);
    for (int c0 = tid * 4; c0 < cols; c0 += ROW_FLY * ROW_THREADS * 4) {
        float v[ROW_FLY][4];
#pragma unroll
        for (int u = 0; u < ROW_FLY; ++u) load_vec<float>(row + min(c0 + u * ROW_THREADS * 4, ld - 4), v[u]);
#pragma unroll
        for (int u = 0; u < ROW_FLY; ++u) {
            const int c = c0 + u * ROW_THREADS * 4;
            float top = LOWEST, sum = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (c + e >= cols) v[u][e] = -INFINITY;
                top = fmaxf(top, v[u][e]);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) sum += __builtin_amdgcn_exp2f((v[u][e] - top) * LOG2E);
            s = join(s, make_float2(top, sum));
        }
    }
    const float top = wave_max(s.x);
    const float sum = wave_sum(s.y * __builtin_amdgcn_exp2f((s.x - top) * LOG2E));
    if (tid % WAVE == 0) part[tid / WAVE] = make_float2(top, sum);
    __syncthreads();
    if (tid) return;
    s = part[0];
#pragma unroll
    for (int i = 1; i < ROW_THREADS / WAVE; ++i) s = join(s, part[i]);
    stats[t] = s;
    const int target = targets[t];
    if (counts(target, vocab) && target >= v0 && target < v0 + cols) at_target[t] = row[target - v0];
}
// dW of up to three columns, which the products' groups of four leave: to (+)= rows^T dz, 32 rows of W a workgroup, 32 threads each, which take every 32nd token
// and are added in order.  A few dependent trips to memory bound it.
constexpr int LAST_FLY = 4;
__global__ __launch_bounds__(1024) void xent_columns_kernel(const float* __restrict__ rows, int hidden, const float* __restrict__ dz, int ldz, int m, int cols,
                                                            float* __restrict__ to, int ldto, int overwrite) {
    __shared__ float part[3][32][33];
    const int i = blockIdx.x * 32 + threadIdx.x % 32, q = threadIdx.x / 32;
    float sum[3] = {0.f, 0.f, 0.f};
    for (int t0 = q; t0 < m; t0 += 32 * LAST_FLY) {
        float x[LAST_FLY], d[LAST_FLY][3];
#pragma unroll
        for (int u = 0; u < LAST_FLY; ++u) {
            const int t = min(t0 + 32 * u, m - 1);
            x[u] = rows[(size_t)t * hidden + min(i, hidden - 1)];
#pragma unroll
            for (int c = 0; c < 3; ++c) d[u][c] = dz[(size_t)t * ldz + min(c, cols - 1)];
        }
#pragma unroll
        for (int u = 0; u < LAST_FLY; ++u)
#pragma unroll
            for (int c = 0; c < 3; ++c) sum[c] += t0 + 32 * u < m ? x[u] * d[u][c] : 0.f;
    }
#pragma unroll
    for (int c = 0; c < 3; ++c) part[c][q][threadIdx.x % 32] = sum[c];
    __syncthreads();
    if (q >= cols || i >= hidden) return;
    float v = 0.f;
    for (int k = 0; k < 32; ++k) v += part[q][k][threadIdx.x % 32];
    float* dst = to + (size_t)i * ldto + q;
    *dst = overwrite ? v : *dst + v;
}

size_t aligned(size_t b) { return (b + 255) / 256 * 256; }
int round_up(int v, int a) { return (v + a - 1) / a * a; }
long tiles_of(int m, int n, int tile) { return (long)((m + tile - 1) / tile) * ((n + tile - 1) / tile); }

// Columns of the forward's product on 256x256 tiles: whole rounds of them, and the rest too where it fills more than half of one; otherwise the rest, which is four
// times as many 128x128 tiles, takes up to two rounds of these, 0.38 each of a large one's time.  2048 tokens, hidden 1600, us with the rest on large tiles and on small:
// 64 tiles over one round 75.8, 57.5; 128 74.6, 69.8; 136 76.4, 81.2; 160 75.5, 80.1; 64 tiles in all 37.2, 18.8; 128 36.1, 32.2; 136 37.5, 43.9; 224 41.3, 56.4;
// and over four rounds 64 191.7, 173.9; 144 191.7, 197.1.  Up to 128 tokens a large tile's step, 2048 clocks of matrix instructions whatever its rows hold, is half
// idle: 128 x 1600 x 20001 38.1, 22.6; x 50257 43.3, 42.7; but 128 x 256 x 50257 18.7, 21.9; and from 129 on 129 x 1600 x 50257 46.7, 70.6.
int wide_columns(int m, int n) {
    const int tm = (m + 255) / 256, tn = (n + 255) / 256;
    const long tiles = (long)tm * tn, over = tiles % NUM_CUS;
    if (tiles <= NUM_CUS / 2 || m <= 128) return 0;
    if (over > NUM_CUS / 2 || over == 0) return tn * 256;
    return (int)((tiles - over) / tm) * 256;
}

// Columns of the vocabulary per piece where the caller leaves it open: 8192, more where a piece's buffers (dz, and bf16 W) stay below 128 MB, fewer where they would
// pass 512 MB, in equal pieces.  There are two sets of them, and dW's parts, where its contraction is cut, come on top.
// From 2048 tokens on, a piece of 8192 columns or somewhat more whose dW just fills the chip's rounds of 256x256 tiles is taken as it is, up to 768 MB, unless that
// leaves a last one of less than a tenth, a pass for little.  Equal pieces -> this, 32 sizes each of hidden 1536 to 2048 and vocabulary 20001 to 128000: 2048 tokens
// 5 % faster to 4 % slower (2048 x 1600 x 50257 1274 -> 1246 us, x 20001 540 -> 558), 4096 8 % to -2 % (4096 x 1600 x 50257 2360 -> 2231), 8192 6 % to -3 %; but 1024
// tokens, where dW is less of the whole, 3 % to -13 % (1024 x 1600 x 65536 900 -> 1035).  Filled pieces below 8192 lose (2048 x 2304 x 65536 in 7168 2100 -> 2266,
// 2048 x 2560 in 6400 2237 -> 2440; but 4096 x 2560 x 50257 3338 -> 3288), beyond 10752 they do from 8192 tokens on (8192 x 1280 x 65536 in 13056 4345 -> 4652, x 1024 in 16384 3493 -> 3627).  Last pieces:
// 2048 x 1600 x 37120 (256 columns behind four of 9216) 936 -> 977, 2048 x 1536 x 44032 (1024 behind four of 10752) 1044 -> 1031.
constexpr size_t PIECE_BYTES_MIN = (size_t)128 << 20, PIECE_BYTES_MAX = (size_t)512 << 20, PIECE_BYTES_FILLED = (size_t)768 << 20;
constexpr int PIECE_STEP = 256, PIECE_USUAL = 8192, PIECE_FILLED_MAX = 10752, PIECE_FILLED_TOKENS = 2048;
int filled_piece(int hidden) {
    const int rows = (hidden + 255) / 256;
    int p = 0;
    for (int rounds = 1; p < PIECE_USUAL; ++rounds) p = NUM_CUS * rounds / rows * 256;
    return p <= PIECE_FILLED_MAX ? p : 0;
}
int default_piece(int dtype, int m, int hidden, int vocab) {
    const int all = round_up(vocab, PIECE_STEP);
    const size_t column = dtype == CHIMERA_F32 ? (size_t)m * 4 : (size_t)round_up(m, TOKEN_PAD) * 8 + (size_t)hidden * 4;
    const size_t usual = std::max(PIECE_BYTES_MIN / column, std::min<size_t>(PIECE_USUAL, PIECE_BYTES_MAX / column));
    const int filled = dtype == CHIMERA_BF16 && m >= PIECE_FILLED_TOKENS && usual <= PIECE_USUAL ? filled_piece(hidden) : 0;
    if (filled && filled < vocab && filled * column <= PIECE_BYTES_FILLED && (vocab % filled == 0 || vocab % filled >= filled / 10)) return filled;
    const int most = (int)std::min<size_t>(all, std::max<size_t>(usual / PIECE_STEP * PIECE_STEP, PIECE_STEP));
    return round_up((vocab + (vocab + most - 1) / most - 1) / ((vocab + most - 1) / most), PIECE_STEP);        // equal pieces
}
// The launches' tiles, and where contractions are cut.  dW on 256x256 tiles where it has half a round of them, or it and dz together a round and a quarter: 64 x 1024, us
// on 128x128 and on 256x256 tiles, 16 columns of large tiles (64 in all) 33.1, 32.4; 30 39.5, 33.5; 34 40.5, 34.0; 300 x 1024, 16 columns 40, 56; 34 61, 63; 40 65, 67; 512 x 256, 120 tiles of both 37.6, 50.4; 1024 x 256, 280 73.8, 71.2; 480 108.7, 85.9;
// 1536 x 256, 280 76.3, 88.0; 336 85.3, 97.3; 504 108.6, 104.3; 672 147.6, 119.4.  Tokens in tiles of 128 up to 128 of them, us beside tiles of 256: 128 x 1600 x 50257
// 285, 320; 128 x 512 x 50257 102, 104; 129 x 512 x 50257 119, 108; 400 x 1600 472, 458; but 129 x 1600 312, 332; 256 x 2048 x 20001 168, 203.
// dh's tiles are cut along the vocabulary
// to half of what a CU has to do in all, or 32 steps, whichever is more (a third and a quarter: 1380 -> 1400 us at 2048 x 1600 x 50256, 360 -> 388 at 512 x 1024,
// every part is read and written once a piece).  dW's are cut along the tokens, to what a CU has to do in all, where one would outlast that by a fifth, as many
// tokens on few columns of h do; their parts are added a pass later (8192 x 256 x 50304 3012 -> 1320 us, 1407 in shorter parts, 1537 uncut in 128x128 tiles;
// 8192 x 768 2994 -> 2540, 2628, 2734; 16384 x 768 10300 -> 5118, 5204, 5593; 4096 x 768 1493 -> 1392, 1489, 1342).
struct PassPlan { int dw_tile, tok_tile, splits, k_per, dw_splits, dw_per; };
PassPlan plan_of(int mp, int hidden, int ld) {
    PassPlan p{};
    const long all256 = tiles_of(hidden, ld, 256) + tiles_of(mp, ld, 256);
    p.dw_tile = tiles_of(hidden, ld, 256) >= 128 || all256 >= 320 ? 256 : 128;
    p.tok_tile = p.dw_tile == 256 && mp > 128 ? 256 : 128;
    auto work = [](int tile, long tiles, long steps) { return tiles * steps * (tile == 256 ? 1.0 : 0.35); };        // in steps of a 256x256 tile
    const long dw_tiles = tiles_of(hidden, ld, p.dw_tile), dw_steps = mp / 32, dh_steps = (ld + 63) / 64, z_steps = (hidden + 63) / 64;
    const double each = (work(p.dw_tile, dw_tiles, dw_steps) + work(p.tok_tile, tiles_of(mp, hidden, p.tok_tile), dh_steps) +
                         work(p.tok_tile, tiles_of(mp, ld, p.tok_tile), z_steps)) / NUM_CUS;
    const double share = p.tok_tile == 256 ? each : each / 0.35;
    const long most = std::max<long>(8, (long)(share < 32 ? share : std::max(32.0, share / 2)));
    const long splits = std::min<long>((dh_steps + most - 1) / most, 64), per = (dh_steps + splits - 1) / splits;
    p.splits = (int)((dh_steps + per - 1) / per);
    p.k_per = (int)per * 64;
    const long rounds = (dw_tiles + NUM_CUS - 1) / NUM_CUS;
    p.dw_per = mp;
    if (work(p.dw_tile, rounds, dw_steps) > 1.2 * each && dw_steps >= 64) {
        const long parts = std::min<long>((long)std::ceil(dw_steps / std::max(32.0, each / work(p.dw_tile, 1, 1))), 16);
        p.dw_per = (int)((dw_steps + parts - 1) / parts) * 32;
    }
    p.dw_splits = (mp + p.dw_per - 1) / p.dw_per;
    return p;
}

struct FwdLayout { int wide, parts; size_t stats, at_target, z, total; int piece; };
FwdLayout fwd_layout(int dtype, int m, int hidden, int vocab) {
    FwdLayout l{};
    size_t b = 0;
    auto take = [&](size_t bytes) { size_t r = b; b += aligned(bytes); return r; };
    l.wide = wide_columns(m, vocab);
    l.piece = default_piece(dtype, m, hidden, vocab);
    l.parts = dtype == CHIMERA_F32 ? (vocab + l.piece - 1) / l.piece : l.wide / 256 + std::max(0, vocab - l.wide + 127) / 128;
    l.stats = take((size_t)l.parts * m * sizeof(float2));
    l.at_target = take((size_t)m * 4);
    l.z = take(dtype == CHIMERA_F32 ? (size_t)m * std::min(l.piece, round_up(vocab, 8)) * 4 : 0);
    l.total = b;
    return l;
}
struct BwdLayout { int piece, ld, mp, ldp, buffers, f32_part; PassPlan plan; size_t room, shift, rows, dz[2], w[2], raise[2], dw[2], slabs, total; };
BwdLayout bwd_layout(int dtype, int m, int hidden, int vocab, int piece) {
    BwdLayout l{};
    size_t b = 0;
    auto take = [&](size_t bytes) { size_t r = b; b += aligned(bytes); return r; };
    l.piece = piece ? round_up(std::min(piece, 1 << 22), PIECE_STEP) : default_piece(dtype, m, hidden, vocab);
    l.ld = std::min(l.piece, round_up(vocab, 8));
    if (dtype == CHIMERA_F32) {
        l.mp = m;
        l.room = take((size_t)m * sizeof(XentRow));
        l.rows = take((size_t)m * hidden * 4);
        l.dz[0] = take((size_t)m * l.ld * 4);
        const int whole = std::max(8, std::min(l.ld, vocab) & ~7);
        l.f32_part = gemm_f32_part(m, hidden, whole);
        l.slabs = take((size_t)((whole + l.f32_part - 1) / l.f32_part) * m * hidden * 4);
    } else {
        l.mp = round_up(m, TOKEN_PAD);
        l.plan = plan_of(l.mp, hidden, l.ld);
        l.ldp = l.ld;
        l.buffers = l.piece < vocab ? 2 : 1;
        l.room = take((size_t)m * 4);
        l.shift = take(4);
        l.rows = take((size_t)l.mp * hidden * 2);
        for (int i = 0; i < l.buffers; ++i) {
            l.dz[i] = take((size_t)l.mp * l.ld * 4);
            l.w[i] = take((size_t)hidden * l.ldp * 2);
            l.raise[i] = take((size_t)hidden * 4);
            l.dw[i] = take(l.plan.dw_splits > 1 ? (size_t)l.plan.dw_splits * hidden * l.ld * 4 : 0);
        }
        l.slabs = take((size_t)l.plan.splits * m * hidden * 4);
    }
    l.total = b;
    return l;
}
struct HeadLayout { size_t h, mean, rstd, loss_rows, lse, dh, scratch, ops, total; };
HeadLayout head_layout(int dtype, int m, int hidden, int vocab, int piece) {
    const size_t e = dtype == CHIMERA_F32 ? 4 : 2;
    HeadLayout l{};
    size_t b = 0;
    auto take = [&](size_t bytes) { size_t r = b; b += aligned(bytes); return r; };
    l.h = take((size_t)m * hidden * e);
    l.mean = take((size_t)m * 4);
    l.rstd = take((size_t)m * 4);
    l.loss_rows = take((size_t)m * 4);
    l.lse = take((size_t)m * 4);
    l.dh = take((size_t)m * hidden * e);
    l.scratch = take(layernorm_bwd_scratch_floats(m, hidden) * 4);
    l.ops = take(std::max(fwd_layout(dtype, m, hidden, vocab).total, bwd_layout(dtype, m, hidden, vocab, piece).total));
    l.total = b;
    return l;
}

#define XENT_TRY(expr) do { int rc__ = (expr); if (rc__) return rc__; } while (0)

int check_xent(int dtype, int tokens, int hidden, int vocab, int ldh, int ldw) {
    if (dtype != CHIMERA_F32 && dtype != CHIMERA_BF16) return fail(CHIMERA_EINVAL, "unknown dtype %d", dtype);
    if (tokens < 1 || hidden < 1 || vocab < 1) return fail(CHIMERA_EINVAL, "sizes must be positive");
    if (tokens > 1 << 22 || hidden > 1 << 15 || vocab > 1 << 22 || (long)tokens * vocab > 1l << 38)
        return fail(CHIMERA_EINVAL, "more than 2^22 tokens, 2^15 hidden or 2^22 vocabulary columns, or 2^38 logits");
    if (hidden % 8) return fail(CHIMERA_EINVAL, "hidden=%d must be a multiple of 8", hidden);
    if (ldh % 8 || ldw % 8) return fail(CHIMERA_EINVAL, "leading dimensions ldh=%d, ldw=%d must be multiples of 8", ldh, ldw);
    if (ldh < hidden || ldw < vocab) return fail(CHIMERA_EINVAL, "leading dimension too small");
    if (ldh >= 1 << 23 || ldw >= 1 << 23) return fail(CHIMERA_EINVAL, "leading dimension of 2^23 or more");
    return CHIMERA_OK;
}

template <typename R> R raster_of(int tile, int rows, int cols, int k, bool bands = true) {
    R r{(rows + tile - 1) / tile, (cols + tile - 1) / tile, 1, 0};
    if (bands) r.band = raster_band(r.tiles_m, r.tiles_n, NUM_CUS, (size_t)cols * k * 2);
    r.group_m = raster_group(r.tiles_m, r.band ? r.band : r.tiles_n, std::min((r.tiles_m * r.tiles_n + 7) / 8, PER_XCD), tile, tile);
    return r;
}

int xent_fwd_bf16(int m, int hidden, int vocab, const bf16_t* h, int ldh, const bf16_t* w, int ldw, const int* targets, const FwdLayout& l, char* ws, hipStream_t s) {
    StatsPass p{h, w, targets, (float2*)(ws + l.stats), (float*)(ws + l.at_target), m, vocab, hidden, ldh, ldw, l.wide, 0, {}, {}};
    int large = 0;
    if (l.wide) { p.r256 = raster_of<StatsPass::Raster>(256, m, std::min(l.wide, vocab), hidden); large = p.r256.tiles_m * p.r256.tiles_n; }
    if (l.wide < vocab) { p.r128 = raster_of<StatsPass::Raster>(128, m, vocab - l.wide, hidden); p.small = p.r128.tiles_m * p.r128.tiles_n; }
    hipLaunchKernelGGL(xent_stats_kernel, dim3(p.small + large), dim3(512), 0, s, p);
    CHIMERA_LAUNCH_CHECK("linear cross-entropy");
    return CHIMERA_OK;
}

template <typename T>
int launch_dh_sum(const float* slabs, int splits, const T* dz, int ldz, const T* w, int ldw, int tail, const int* targets, const float* dloss, float scale, int vocab,
                  int m, int n, T* dh, int lddh, hipStream_t s) {
    const size_t threads = (size_t)m * (n / 4);
    hipLaunchKernelGGL(xent_dh_sum_kernel<T>, dim3((unsigned)std::min<size_t>((threads + ROW_THREADS - 1) / ROW_THREADS, 1 << 20)), dim3(ROW_THREADS), 0, s, slabs, splits, dz, ldz, w, ldw, tail,
                       targets, dloss, scale, vocab, m, n, dh, lddh);
    CHIMERA_LAUNCH_CHECK("linear cross-entropy");
    return CHIMERA_OK;
}

int xent_fwd_f32(int m, int hidden, int vocab, const float* h, int ldh, const float* w, int ldw, const int* targets, const FwdLayout& l, char* ws, void* stream) {
    for (int v0 = 0, p = 0; v0 < vocab; v0 += l.piece, ++p) {
        const int cols = std::min(l.piece, vocab - v0), ld = round_up(cols, 4);      // (a row of W ends no sooner: 16-byte alignment, leading dimensions in multiples of 8)
        GemmArgs g{};
        g.m = m; g.n = ld; g.k = hidden; g.a = h; g.lda = ldh; g.a_kc = 1; g.b = w + v0; g.ldb = ldw; g.b_kc = 0; g.c = ws + l.z; g.epilogue = EPI_NONE;
        XENT_TRY(gemm_f32(g, stream));
        hipLaunchKernelGGL(xent_stats_f32_kernel, dim3(m), dim3(ROW_THREADS), 0, (hipStream_t)stream, (const float*)(ws + l.z), ld, cols, v0, vocab, targets,
                           (float2*)(ws + l.stats) + (size_t)p * m, (float*)(ws + l.at_target));
        CHIMERA_LAUNCH_CHECK("linear cross-entropy");
    }
    return CHIMERA_OK;
}

int xent_bwd_f32(int m, int hidden, int vocab, const float* h, int ldh, const float* w, int ldw, const int* targets, const float* lse, float scale,
                 const float* dloss, float* dh, int lddh, float* dw, int lddw, int overwrite, const BwdLayout& l, char* ws, void* stream) {
    hipStream_t s = (hipStream_t)stream;
    float *rows = (float*)(ws + l.rows), *z = (float*)(ws + l.dz[0]), *slab = (float*)(ws + l.slabs);
    XentRow* info = (XentRow*)(ws + l.room);
    hipLaunchKernelGGL(xent_rows_f32_kernel, dim3((m + 3) / 4), dim3(ROW_THREADS), 0, s, h, ldh, targets, lse, dloss, scale, m, hidden, vocab, info, dw ? rows : nullptr);
    CHIMERA_LAUNCH_CHECK("linear cross-entropy");
    int slabs = 0;
    for (int v0 = 0; v0 < vocab; v0 += l.piece) {
        const int cols = std::min(l.piece, vocab - v0), ld = round_up(cols, 4), whole = cols & ~7;
        GemmArgs g{};
        g.m = m; g.n = ld; g.k = hidden; g.a = h; g.lda = ldh; g.a_kc = 1; g.b = w + v0; g.ldb = ldw; g.b_kc = 0; g.c = z;
        g.epilogue = EPI_XENT; g.bias = info; g.gelu_erf = v0;
        XENT_TRY(gemm_f32(g, stream));
        if (dh && whole) {
            GemmArgs d{};
            d.m = m; d.n = hidden; d.k = whole; d.a = z; d.lda = ld; d.a_kc = 1; d.b = w + v0; d.ldb = ldw; d.b_kc = 1; d.c = slab;
            d.epilogue = slabs ? EPI_ACCUM_F32 : EPI_NONE;
            XENT_TRY(gemm_f32_parts(d, l.f32_part, (size_t)m * hidden, stream));       // (a last piece is cut where the others are, and may have fewer parts)
            if (!slabs) slabs = (whole + l.f32_part - 1) / l.f32_part;
        }
        if (dw) {
            const int fours = cols & ~3;
            GemmArgs q{};
            q.m = hidden; q.n = fours; q.k = m; q.a = rows; q.lda = hidden; q.a_kc = 0; q.b = z; q.ldb = ld; q.b_kc = 0; q.c = dw + v0; q.ldc = lddw;
            q.epilogue = EPI_ACCUM_F32;
            if (fours) XENT_TRY(gemm_f32_group(1, &q, nullptr, overwrite, stream));
            if (fours < cols)
                hipLaunchKernelGGL(xent_columns_kernel, dim3((hidden + 31) / 32), dim3(1024), 0, s, rows, hidden, z + fours, ld, m, cols - fours, dw + v0 + fours, lddw,
                                   overwrite);
            CHIMERA_LAUNCH_CHECK("linear cross-entropy");
        }
        if (dh && v0 + l.piece >= vocab) {
            XENT_TRY(launch_dh_sum(slab, slabs, z + whole, ld, w + v0 + whole, ldw, cols - whole, targets, dloss, scale, vocab, m, hidden, dh, lddh, s));
        }
    }
    return CHIMERA_OK;
}

int xent_bwd_bf16(int m, int hidden, int vocab, const bf16_t* h, int ldh, const bf16_t* w, int ldw, const int* targets, const float* lse, float scale,
                  const float* dloss, bf16_t* dh, int lddh, float* dw, int lddw, int overwrite, const BwdLayout& l, char* ws, void* stream) {
    hipStream_t s = (hipStream_t)stream;
    Pass p{};
    p.h = h; p.w = w; p.targets = targets; p.lse = lse; p.dloss = dloss; p.scale = scale;
    p.m = m; p.mp = l.mp; p.hidden = hidden; p.vocab = vocab; p.ldh = ldh; p.ldw = ldw; p.ldp = l.ldp;
    p.room = (int*)(ws + l.room); p.shift = (int*)(ws + l.shift); p.rows = (_Float16*)(ws + l.rows);
    p.dw = dw; p.lddw = lddw; p.dw_flags = overwrite ? ACCUM_OVERWRITE : 0;
    p.slabs = (float*)(ws + l.slabs); p.k_per = l.plan.k_per; p.dw_per = l.plan.dw_per; p.dw_splits = l.plan.dw_splits;
    p.w_rows = 8;                                          // fewer where that leaves few workgroups
    while (p.w_rows > 1 && hidden / p.w_rows < 128) p.w_rows /= 2;
    if (dw) {
        hipLaunchKernelGGL(xent_room_kernel, dim3((m + 3) / 4), dim3(ROW_THREADS), 0, s, h, ldh, targets, dloss, scale, m, hidden, vocab, p.room);
        CHIMERA_LAUNCH_CHECK("linear cross-entropy");
    }
    const int pieces = (vocab + l.piece - 1) / l.piece;
    int splits = 0;
    const bool cut = dw && l.plan.dw_splits > 1;
    for (int i = 0; i <= pieces + cut; ++i) {
        p.past = p.now;
        p.now = p.next;
        int (&count)[6] = p.count;
        std::fill(std::begin(count), std::end(count), 0);
        if (cut && i > 1) count[5] = (int)std::min<size_t>(((size_t)hidden * p.past.ld / 4 + 511) / 512, SUM_WGS);
        if (i > 0 && i <= pieces) {
            if (dw) {
                p.dw_r = raster_of<Pass::Raster>(l.plan.dw_tile, hidden, p.now.ld, 2 * l.mp);
                count[0] = p.dw_r.tiles_m * p.dw_r.tiles_n * l.plan.dw_splits;
            }
            if (dh) {
                // the last piece is cut where the others are: a split that it does not reach adds nothing
                const int now = (p.now.ld + l.plan.k_per - 1) / l.plan.k_per;
                p.dh_r = raster_of<Pass::Raster>(l.plan.tok_tile, m, hidden, 0, false);
                count[1] = p.dh_r.tiles_m * p.dh_r.tiles_n * now;
                p.dh_flags = i == 1 ? ACCUM_OVERWRITE : 0;
                if (i == 1) splits = now;
            }
        }
        if (i < pieces) {
            const int v0 = i * l.piece, cols = std::min(l.piece, vocab - v0), at = i & (l.buffers - 1);
            p.next = {v0, cols, round_up(cols, 8), (_Float16*)(ws + l.dz[at]), (_Float16*)(ws + l.w[at]), (int*)(ws + l.raise[at]),
                      (float*)(ws + l.dw[at])};
            p.dz_r = raster_of<Pass::Raster>(l.plan.tok_tile, l.mp, p.next.ld, hidden);
            count[2] = p.dz_r.tiles_m * p.dz_r.tiles_n;
            if (dh) count[3] = (hidden + p.w_rows - 1) / p.w_rows;
            if (dw && i == 0) count[4] = (int)std::min<long>((long)((l.mp + TURN_TOKENS - 1) / TURN_TOKENS) * ((hidden + TURN_COLS - 1) / TURN_COLS), TURN_WGS);
        }
        // The longest first.  Where dz has few tiles these are the rows, which wait for memory (1 x 128 x 44312 64 -> 39 us; but 8192 x 2048 x 32768, 1024 tiles,
        // 3555 -> 3585).
        const bool rows_first = i == 0 && count[2] <= 2 * NUM_CUS;
        int total = 0;
        for (int k : rows_first ? std::array{4, 3, 2, 1, 0, 5} : std::array{0, 1, 2, 3, 4, 5}) { p.first[k] = total; total += count[k]; }
        if (l.plan.dw_tile == 256 && l.plan.tok_tile == 256) hipLaunchKernelGGL((xent_pass_kernel<256, 256>), dim3(total), dim3(512), 0, s, p);
        else if (l.plan.dw_tile == 256) hipLaunchKernelGGL((xent_pass_kernel<256, 128>), dim3(total), dim3(512), 0, s, p);
        else hipLaunchKernelGGL((xent_pass_kernel<128, 128>), dim3(total), dim3(512), 0, s, p);
        CHIMERA_LAUNCH_CHECK("linear cross-entropy");
    }
    return dh ? launch_dh_sum<bf16_t>(p.slabs, splits, nullptr, 0, nullptr, 0, 0, targets, dloss, scale, vocab, m, hidden, dh, lddh, s) : CHIMERA_OK;
}

}  // namespace
}  // namespace chimera

using namespace chimera;

extern "C" {

size_t chimera_op_linear_xent_fwd_workspace_bytes(int dtype, int tokens, int hidden, int vocab) {
    return check_xent(dtype, tokens, hidden, vocab, hidden, round_up(std::max(vocab, 1), 8)) ? 0 : fwd_layout(dtype, tokens, hidden, vocab).total;
}

size_t chimera_op_linear_xent_bwd_workspace_bytes(int dtype, int tokens, int hidden, int vocab, int piece) {
    if (piece < 0 || check_xent(dtype, tokens, hidden, vocab, hidden, round_up(std::max(vocab, 1), 8))) return 0;
    return bwd_layout(dtype, tokens, hidden, vocab, piece).total;
}

int chimera_op_linear_xent_fwd(int dtype, int tokens, int hidden, int vocab, const void* d_h, int ldh, const void* d_w, int ldw, const int32_t* d_targets,
                               float scale, float* d_loss_rows, float* d_lse, float* d_loss, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
    XENT_TRY(check_xent(dtype, tokens, hidden, vocab, ldh, ldw));
    if (!d_h || !d_w || !d_targets || !d_loss_rows || !d_lse || !d_workspace) return fail(CHIMERA_EINVAL, "NULL operand");
    if (((uintptr_t)d_workspace & 255) || (((uintptr_t)d_h | (uintptr_t)d_w) & 15)) return fail(CHIMERA_EINVAL, "workspace must be 256-byte aligned, tensors 16-byte aligned");
    const FwdLayout l = fwd_layout(dtype, tokens, hidden, vocab);
    if (workspace_bytes < l.total) return fail(CHIMERA_ENOMEM, "workspace holds %zu bytes, need %zu", workspace_bytes, l.total);
    const size_t e = dtype == CHIMERA_F32 ? 4 : 2, m = (size_t)tokens;
    XENT_TRY(check_apart({matrix(d_h, m, hidden, ldh, e), matrix(d_w, hidden, vocab, ldw, e), plain(d_targets, m * 4)},
                         {plain(d_loss_rows, m * 4), plain(d_lse, m * 4), plain(d_loss, 4), plain(d_workspace, l.total)}));
    char* ws = (char*)d_workspace;
    float2* stats = (float2*)(ws + l.stats);
    float* at_target = (float*)(ws + l.at_target);
    hipStream_t s = (hipStream_t)hip_stream;
    if (dtype == CHIMERA_F32)
        XENT_TRY(xent_fwd_f32(tokens, hidden, vocab, (const float*)d_h, ldh, (const float*)d_w, ldw, d_targets, l, ws, hip_stream));
    else
        XENT_TRY(xent_fwd_bf16(tokens, hidden, vocab, (const bf16_t*)d_h, ldh, (const bf16_t*)d_w, ldw, d_targets, l, ws, s));
    if (tokens <= JOIN_ALONE) {
        hipLaunchKernelGGL(xent_join_kernel<WAVE>, dim3(1), dim3(16 * WAVE), 0, s, stats, at_target, d_targets, tokens, vocab, l.parts, scale, d_loss_rows, d_lse, d_loss);
        CHIMERA_LAUNCH_CHECK("linear cross-entropy");
        return CHIMERA_OK;
    }
    hipLaunchKernelGGL(xent_join_kernel<16>, dim3((tokens + 15) / 16), dim3(256), 0, s, stats, at_target, d_targets, tokens, vocab, l.parts, scale, d_loss_rows, d_lse,
                       nullptr);
    CHIMERA_LAUNCH_CHECK("linear cross-entropy");
    return d_loss ? loss_sum(d_loss_rows, tokens, d_loss, hip_stream) : CHIMERA_OK;
}

int chimera_op_linear_xent_bwd(int dtype, int tokens, int hidden, int vocab, const void* d_h, int ldh, const void* d_w, int ldw, const int32_t* d_targets,
                               const float* d_lse, float scale, const float* d_dloss, void* d_dh, int lddh, float* d_dw, int lddw, int overwrite, int piece,
                               void* d_workspace, size_t workspace_bytes, void* hip_stream) {
    XENT_TRY(check_xent(dtype, tokens, hidden, vocab, ldh, ldw));
    if (!d_h || !d_w || !d_targets || !d_lse || !d_workspace) return fail(CHIMERA_EINVAL, "NULL operand");
    if (!d_dh && !d_dw) return fail(CHIMERA_EINVAL, "neither dh nor dw is asked for");
    if (piece < 0) return fail(CHIMERA_EINVAL, "piece=%d is negative", piece);
    if (d_dh && (lddh < hidden || lddh % 8)) return fail(CHIMERA_EINVAL, "lddh=%d must be a multiple of 8 and at least hidden=%d", lddh, hidden);
    if (d_dw && (lddw < vocab || lddw % 8)) return fail(CHIMERA_EINVAL, "lddw=%d must be a multiple of 8 and at least vocab=%d", lddw, vocab);
    if (((uintptr_t)d_workspace & 255) || (((uintptr_t)d_h | (uintptr_t)d_w | (uintptr_t)d_dh | (uintptr_t)d_dw) & 15))
        return fail(CHIMERA_EINVAL, "workspace must be 256-byte aligned, tensors 16-byte aligned");
    const BwdLayout l = bwd_layout(dtype, tokens, hidden, vocab, piece);
    if (workspace_bytes < l.total) return fail(CHIMERA_ENOMEM, "workspace holds %zu bytes, need %zu", workspace_bytes, l.total);
    const size_t e = dtype == CHIMERA_F32 ? 4 : 2, m = (size_t)tokens;
    const Rows dh = matrix(d_dh, m, hidden, lddh, e), dw = matrix(d_dw, hidden, vocab, lddw, 4), h = matrix(d_h, m, hidden, ldh, e), rest = plain(d_workspace, l.total);
    // (dh is written when h has been read for the last time, and may take its place)
    for (const Rows& r : {matrix(d_w, hidden, vocab, ldw, e), plain(d_targets, m * 4), plain(d_lse, m * 4), plain(d_dloss, m * 4)}) XENT_TRY(check_apart({r}, {dh, dw, rest}));
    XENT_TRY(check_apart({h}, {dw, rest}));
    char* ws = (char*)d_workspace;
    if (dtype == CHIMERA_F32)
        return xent_bwd_f32(tokens, hidden, vocab, (const float*)d_h, ldh, (const float*)d_w, ldw, d_targets, d_lse, scale, d_dloss, (float*)d_dh, lddh, d_dw, lddw,
                            overwrite, l, ws, hip_stream);
    return xent_bwd_bf16(tokens, hidden, vocab, (const bf16_t*)d_h, ldh, (const bf16_t*)d_w, ldw, d_targets, d_lse, scale, d_dloss, (bf16_t*)d_dh, lddh, d_dw, lddw,
                         overwrite, l, ws, hip_stream);
}

size_t chimera_head_pieces_workspace_bytes(int dtype, int tokens, int hidden, int vocab, int piece) {
    if (piece < 0 || check_xent(dtype, tokens, hidden, vocab, hidden, round_up(std::max(vocab, 1), 8))) return 0;
    return head_layout(dtype, tokens, hidden, vocab, piece).total;
}

int chimera_head_loss_pieces(int dtype, int tokens, int hidden, int vocab, const void* d_y, const int32_t* d_targets, const void* d_lnf_g, const void* d_lnf_b,
                             const void* d_w_head, int ldw, float scale, void* d_dy, float* d_dlnf_g, float* d_dlnf_b, float* d_dw_head, float* d_loss, int piece,
                             void* d_workspace, size_t workspace_bytes, void* hip_stream) {
    XENT_TRY(check_xent(dtype, tokens, hidden, vocab, hidden, ldw));
    if (!d_y || !d_targets || !d_lnf_g || !d_lnf_b || !d_w_head || !d_dy || !d_dlnf_g || !d_dlnf_b || !d_dw_head || !d_loss || !d_workspace)
        return fail(CHIMERA_EINVAL, "NULL operand");
    if (piece < 0) return fail(CHIMERA_EINVAL, "piece=%d is negative", piece);
    if (((uintptr_t)d_workspace & 255) || (((uintptr_t)d_y | (uintptr_t)d_dy | (uintptr_t)d_w_head | (uintptr_t)d_dw_head) & 15))
        return fail(CHIMERA_EINVAL, "workspace must be 256-byte aligned, tensors 16-byte aligned");
    const HeadLayout l = head_layout(dtype, tokens, hidden, vocab, piece);
    if (workspace_bytes < l.total) return fail(CHIMERA_ENOMEM, "workspace holds %zu bytes, need %zu", workspace_bytes, l.total);
    const size_t e = dtype == CHIMERA_F32 ? 4 : 2, m = (size_t)tokens, v = (size_t)hidden;
    const Rows dy = plain(d_dy, m * v * e), dg = plain(d_dlnf_g, v * 4), db = plain(d_dlnf_b, v * 4), dw = matrix(d_dw_head, v, vocab, ldw, 4), loss = plain(d_loss, 4),
               rest = plain(d_workspace, l.total);
    // (dy is written last, where each row of y has just been read, and may be y itself)
    XENT_TRY(check_apart({matrix(d_w_head, v, vocab, ldw, e), plain(d_targets, m * 4), plain(d_lnf_g, v * e), plain(d_lnf_b, v * e)}, {dy, dg, db, dw, loss, rest}));
    XENT_TRY(check_apart({plain(d_y, m * v * e)}, {d_dy == d_y ? plain(nullptr, 1) : dy, dg, db, dw, loss, rest}));
    char* ws = (char*)d_workspace;
    void *h = ws + l.h, *dh = ws + l.dh;
    float *mean = (float*)(ws + l.mean), *rstd = (float*)(ws + l.rstd), *rows = (float*)(ws + l.loss_rows), *lse = (float*)(ws + l.lse);
    XENT_TRY(layernorm_fwd(dtype, tokens, hidden, d_y, 0, d_lnf_g, d_lnf_b, h, mean, rstd, hip_stream));
    XENT_TRY(chimera_op_linear_xent_fwd(dtype, tokens, hidden, vocab, h, hidden, d_w_head, ldw, d_targets, scale, rows, lse, d_loss, ws + l.ops, l.total - l.ops, hip_stream));
    XENT_TRY(chimera_op_linear_xent_bwd(dtype, tokens, hidden, vocab, h, hidden, d_w_head, ldw, d_targets, lse, scale, nullptr, dh, hidden, d_dw_head, ldw, 0, piece,
                                        ws + l.ops, l.total - l.ops, hip_stream));
    return layernorm_bwd(dtype, tokens, hidden, dh, d_y, 0, mean, rstd, d_lnf_g, nullptr, 0, d_dy, nullptr, d_dlnf_g, d_dlnf_b, (float*)(ws + l.scratch), 0, hip_stream);
}

}  // extern "C"
