// Vocabulary projection and softmax cross-entropy without the logits, forward and backward:
//   z = h W (h [M, H], W stored [H, V]),  lse_t = log sum_v exp z_tv,  loss_t = scale (lse_t - z_t,target)
//   dz_tv = coef_t (exp(z_tv - lse_t) - [v = target_t]),  coef_t = scale dloss_t,  dh = dz W^T,  dW (+)= h^T dz
// A token whose target lies outside [0, V) does not count: loss 0, coef 0, whatever its hidden state holds.
//
// bf16.  The forward's product ends in the statistics of its tile instead of in z: a (maximum, sum) pair per row and tile,
// which a second kernel combines.  The backward forms z again, a piece of the vocabulary at a time, and ends in dz of
// that piece; two products take it from there, and the next piece takes its place.
// dz goes into dW as two fp16 numbers, because dW is a float sum: one bf16 dz would leave it 2e-3 off, two 3e-6, two of fp16
// (11 bits each) 1e-7.  fp16 holds h, a bf16 number, exactly only within its range, so every row of h is scaled by a power of two,
// 2^up_t, that puts its largest number into [2^14, 2^15), where fp16 loses nothing above 2^-28 of it; dz_t takes 2^(shift - up_t), with the
// largest `shift` that keeps all of dz below 2^15, and dW's epilogue takes 2^-shift off again.
// dh is rounded to bf16 itself, and takes dz as one bf16 number.
//
// float.  The framework's float products on pieces of z that are in memory, row kernels between them.
#include "gemm_tiles.h"

#include <climits>

namespace chimera {
namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LOWEST = -3.0e38f;              // stands for the maximum of nothing: differences from it stay finite
constexpr int TOKEN_PAD = 32;                   // the weight gradient's contraction, two rows a token, is walked in steps of 64
constexpr int ROW_THREADS = 256;

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
    float2* stats;               // [tile column][token]
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

template <int BM, int BN, int WGM, int WGN, int WGK>
__global__ __launch_bounds__(WGM* WGN * WGK * 64, 2) void xent_stats_kernel(
    const bf16_t* __restrict__ h, const bf16_t* __restrict__ w, const int* __restrict__ targets, float2* __restrict__ stats,
    float* __restrict__ at_target, int m, int vocab, int k, int ldh, int ldw, int tiles_m, int tiles_n, int group_m, int band) {
    __shared__ __attribute__((aligned(1024))) char lds[RingLds<BM, BN, WGM, WGN, WGK>::BYTES];
    gemm_ring_tile<BM, BN, WGM, WGN, WGK, true, false, EPI_OWN>(lds, h, w, nullptr, nullptr, nullptr, nullptr, m, (vocab + 7) & ~7, k, ldh, ldw, EPI_OWN, 0, 0,
                                                                tiles_m, tiles_n, group_m, (int)blockIdx.x, nullptr, true, 0, Ahead{nullptr, 0}, band,
                                                                StatsEnd<BM, BN>{targets, stats, at_target, m, vocab});
}

// The pairs of a row, joined: 16 rows a workgroup, 16 lanes each, which take every sixteenth pair and join theirs in order.
__global__ __launch_bounds__(256) void xent_join_kernel(const float2* __restrict__ stats, const float* __restrict__ at_target, const int* __restrict__ targets,
                                                        int m, int vocab, int parts, float scale, float* __restrict__ loss_rows, float* __restrict__ lse) {
    __shared__ float2 tab[16][16];
    const int r = threadIdx.x & 15, q = threadIdx.x >> 4, row = blockIdx.x * 16 + r;
    float2 s = make_float2(LOWEST, 0.f);
    if (row < m)
        for (int p = q; p < parts; p += 16) s = join(s, stats[(size_t)p * m + row]);
    tab[q][r] = s;
    __syncthreads();
    if (q || row >= m) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) s = join(s, tab[i][r]);
    const float l = s.x + logf(s.y);
    lse[row] = l;
    loss_rows[row] = counts(targets[row], vocab) ? scale * (l - at_target[row]) : 0.f;
}

// ---- backward: the rows of h that the weight gradient takes, tokens that do not count (and the padding behind the last one) as zeros: their dz is
// zero, but h may hold anything.  bf16: fp16 numbers times 2^up, written twice, once for either half of dz, and the largest
// shift that this row allows (INT_MAX: any).  One wavefront per row.
template <typename T, typename U>
__global__ __launch_bounds__(ROW_THREADS) void xent_rows_kernel(const T* __restrict__ h, int ldh, const int* __restrict__ targets, const float* __restrict__ dloss,
                                                                float scale, int m, int mp, int cols, int vocab, U* __restrict__ out, int* __restrict__ up,
                                                                int* __restrict__ room) {
    constexpr int V = Elem<T>::VEC;
    const int t = blockIdx.x * (ROW_THREADS / WAVE) + threadIdx.x / WAVE, lane = threadIdx.x % WAVE;
    if (t >= mp) return;
    const float coef = t < m && counts(targets[t], vocab) ? (dloss ? scale * dloss[t] : scale) : 0.f;
    const T* src = h + (size_t)min(t, m - 1) * ldh;
    int lift = 0;
    if constexpr (sizeof(U) == 2) {
        float top = 0.f;
        if (coef != 0.f)
            for (int c = lane; c < cols / V; c += WAVE) {
                float x[V];
                load_vec<T>(src + c * V, x);
#pragma unroll
                for (int e = 0; e < V; ++e) top = fmaxf(top, fabsf(x[e]));
            }
        top = wave_max(top);
        lift = top > 0.f ? 15 - __builtin_amdgcn_frexp_expf(top) : 0;       // top = f 2^exp, f in [1/2, 1)
        // |dz| <= |coef| = f 2^exp, and one bit to spare
        if (lane == 0 && t < m) { up[t] = lift; room[t] = top > 0.f && coef != 0.f ? lift + 14 - __builtin_amdgcn_frexp_expf(coef) : INT_MAX; }
    }
    for (int c = lane; c < cols / V; c += WAVE) {
        float x[V];
        load_vec<T>(src + c * V, x);
        U* to = out + (size_t)t * cols + c * V;
        if constexpr (sizeof(U) == 2) {
            f16x8 y;
#pragma unroll
            for (int e = 0; e < V; ++e) y[e] = coef != 0.f ? (_Float16)ldexpf(x[e], lift) : (_Float16)0.f;
            *reinterpret_cast<f16x8*>(to) = y;
            *reinterpret_cast<f16x8*>(to + (size_t)mp * cols) = y;
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) x[e] = coef != 0.f ? x[e] : 0.f;
            store_vec<U>(to, x);
        }
    }
}
// The largest shift that every row allows.
__global__ __launch_bounds__(1024) void xent_shift_kernel(const int* __restrict__ room, int m, int* __restrict__ shift) {
    __shared__ int part[16];
    int v = INT_MAX;
    for (int t = threadIdx.x; t < m; t += 1024) v = min(v, room[t]);
#pragma unroll
    for (int o = 32; o; o >>= 1) v = min(v, __shfl_xor(v, o, WAVE));
    if (threadIdx.x % WAVE == 0) part[threadIdx.x / WAVE] = v;
    __syncthreads();
    if (threadIdx.x) return;
    for (int i = 1; i < 16; ++i) v = min(v, part[i]);
    *shift = v == INT_MAX ? 0 : v;
}

// ---- what the backward's tiles of z end in: dz of the piece, as one bf16 number for dh and as two of fp16 for dW
struct RowInfo { float lse, coef, scaled; int at; };        // at: the target's column in the piece
template <int BM, int SLABS> struct GradEnd {
    const float* lse;
    const int* targets;
    const float* dloss;
    const int *up, *shift;
    float scale;
    int m, mp, vocab, v0, cols, ld;                         // tokens (padded to mp); the piece's first column, its columns, the rows of dz
    bf16_t* dz;                                             // [mp, ld]
    _Float16* parts;                                        // [2 mp, ld]
    RowInfo mine;
    __device__ __forceinline__ void begin(int i0, int tid) {
        // (no branches: the compiler keeps the tile's operand addresses in scalar registers only outside of divergent code)
        const int t = min(i0 + tid, m - 1), target = targets[t];
        const bool on = i0 + tid < m && counts(target, vocab);
        const float coef = on ? (dloss ? scale * dloss[t] : scale) : 0.f;
        mine = {lse[t], coef, ldexpf(coef, *shift - up[t]), on ? target - v0 : -1};
    }
    template <int TO, int TN2, typename Acc>
    __device__ __forceinline__ void end(const Acc& out, char* lds, int i0, int rb0, int cb0, int, int wave, int lane) const {
        constexpr int CPR = EpiSlab<TN2>::WN / 8, RPP = 64 / CPR, NP = 32 / RPP;
        RowInfo* tab = reinterpret_cast<RowInfo*>(lds + SLABS * EpiSlab<TN2>::FLOATS * sizeof(float));
        float* slab = reinterpret_cast<float*>(lds) + (size_t)wave * EpiSlab<TN2>::FLOATS;
        const int tid = threadIdx.x;
        if (tid < BM) tab[tid] = mine;
        __syncthreads();
        const int pr = lane / CPR, pc = lane % CPR * 8, col = cb0 + pc;
        static_for<TO>([&](auto a_c) {
            constexpr int a = decltype(a_c)::value;
            out.template put<a>(slab, lane);
            __builtin_amdgcn_s_waitcnt(0xc07f);                   // lgkmcnt(0): the slab is written (wavefront-private)
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int j = 0; j < NP; ++j) {
                const int lr = a * 32 + j * RPP + pr, row = rb0 + lr;
                const RowInfo r = tab[rb0 - i0 + lr];
                float v[8];
                load_vec<float>(EpiSlab<TN2>::at(slab, j * RPP + pr, pc / 4), v);
                load_vec<float>(EpiSlab<TN2>::at(slab, j * RPP + pr, pc / 4 + 1), v + 4);
                if (row >= mp || col >= ld) continue;
                f16x8 hi, lo;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float d = __builtin_amdgcn_exp2f((v[e] - r.lse) * LOG2E) - (col + e == r.at ? 1.0f : 0.0f);
                    if (r.coef == 0.f || col + e >= cols) d = 0.f;
                    v[e] = r.coef * d;
                    const float x = r.scaled * d;
                    hi[e] = (_Float16)x;
                    lo[e] = (_Float16)(x - (float)hi[e]);
                }
                const size_t at = (size_t)row * ld + col;
                store_vec<bf16_t>(dz + at, v);
                *reinterpret_cast<f16x8*>(parts + at) = hi;
                *reinterpret_cast<f16x8*>(parts + (size_t)mp * ld + at) = lo;
            }
            __builtin_amdgcn_wave_barrier();                      // all lanes have read the slab before it is rewritten
        });
    }
};

template <int BM, int BN, int WGM, int WGN, int WGK>
__global__ __launch_bounds__(WGM* WGN * WGK * 64, 2) void xent_dz_kernel(
    const bf16_t* __restrict__ h, const bf16_t* __restrict__ w, int k, int ldh, int ldw, int tiles_m, int tiles_n, int group_m, int band,
    GradEnd<BM, WGM * WGN * WGK> end) {
    __shared__ __attribute__((aligned(1024))) char lds[RingLds<BM, BN, WGM, WGN, WGK>::BYTES];
    static_assert(sizeof lds >= WGM * WGN * WGK * EpiSlab<BN / WGN / 32>::FLOATS * sizeof(float) + BM * sizeof(RowInfo), "room for the slabs and the rows");
    gemm_ring_tile<BM, BN, WGM, WGN, WGK, true, false, EPI_OWN>(lds, h, w + end.v0, nullptr, nullptr, nullptr, nullptr, end.m, end.ld, k, ldh, ldw, EPI_OWN, 0, 0,
                                                                tiles_m, tiles_n, group_m, (int)blockIdx.x, nullptr, true, 0, Ahead{nullptr, 0}, band, end);
}

// ---- dh: float slabs [split][m, n] (+)= dz W^T over the splits of a piece's columns
template <int BM, int BN, int WGM, int WGN, int WGK>
__global__ __launch_bounds__(WGM* WGN * WGK * 64, 2) void xent_dh_kernel(
    const bf16_t* __restrict__ dz, const bf16_t* __restrict__ w, float* __restrict__ slabs, int m, int n, int k, int ldz, int ldw, int tiles_m, int tiles_n,
    int group_m, int splits, int k_per, int flags) {
    const int tiles = tiles_m * tiles_n, total = tiles * splits;
    const int xcd = (int)blockIdx.x & 7, local = (int)blockIdx.x >> 3;
    const int pid = xcd * (total >> 3) + min(xcd, total & 7) + local;
    const int split = __builtin_amdgcn_readfirstlane(pid / tiles), k0 = split * k_per;
    __shared__ __attribute__((aligned(1024))) char lds[RingLds<BM, BN, WGM, WGN, WGK>::BYTES];
    gemm_ring_tile<BM, BN, WGM, WGN, WGK, true, true, EPI_ACCUM_F32>(lds, dz + k0, w + k0, nullptr, nullptr, slabs + (size_t)split * m * n, nullptr, m, n,
                                                                     min(k_per, k - k0), ldz, ldw, EPI_ACCUM_F32, flags, 0, tiles_m, tiles_n, group_m,
                                                                     pid - split * tiles, nullptr, false);
}

// dh = the slabs' sum, and the product of the last vocabulary columns, fewer than 8, that no slab holds: what lies beside them in
// W's rows does not count and need not be a number.  A thread owns 4 columns, a workgroup ROWS tokens.
constexpr int DH_ROWS = 8;
template <typename T>
__global__ __launch_bounds__(ROW_THREADS) void xent_dh_sum_kernel(const float* __restrict__ slabs, int splits, const T* __restrict__ dz, int ldz,
                                                                  const T* __restrict__ w, int ldw, int tail, int m, int n, T* __restrict__ dh, int lddh) {
    const int c = (blockIdx.y * ROW_THREADS + threadIdx.x) * 4;
    if (c >= n) return;
    float wt[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) wt[i][j] = 0.f;
    if (tail) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            load_elems<T, 8>(w + (size_t)(c + i) * ldw, wt[i]);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j >= tail) wt[i][j] = 0.f;
        }
    }
    for (int t = blockIdx.x * DH_ROWS; t < min((int)(blockIdx.x + 1) * DH_ROWS, m); ++t) {
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        for (int s = 0; s < splits; ++s) {
            float u[4];
            load_vec<float>(slabs + ((size_t)s * m + t) * n + c, u);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] += u[i];
        }
        if (tail) {
            float d[8];
            load_elems<T, 8>(dz + (size_t)t * ldz, d);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i] += d[j] * wt[i][j];
        }
        T* to = dh + (size_t)t * lddh + c;
        if constexpr (sizeof(T) == 4) {
            store_vec<float>(to, v);
        } else {
            typedef bf16_t bf16x4_t __attribute__((ext_vector_type(4)));
            *reinterpret_cast<bf16x4_t*>(to) = bf16x4_t{(bf16_t)v[0], (bf16_t)v[1], (bf16_t)v[2], (bf16_t)v[3]};
        }
    }
}

// ---- dW: a piece's columns (+)= h^T dz, 2^shift taken off
struct ColumnsEnd {
    float* c;
    const int* shift;
    int m, n, ldc, flags;
    __device__ __forceinline__ void begin(int, int) {}
    template <int TO, int TN2, typename Acc>
    __device__ __forceinline__ void end(const Acc& out, char* lds, int, int rb0, int cb0, int, int wave, int lane) const {
        float* slab = reinterpret_cast<float*>(lds) + (size_t)wave * EpiSlab<TN2>::FLOATS;
        accumulate<false, true, TO, TN2>(out, slab, rb0, cb0, m, n, ldc, *shift, c, flags, lane);
    }
};
template <int BM, int BN, int WGM, int WGN, int WGK>
__global__ __launch_bounds__(WGM* WGN * WGK * 64, 2) void xent_dw_kernel(const _Float16* __restrict__ h, const _Float16* __restrict__ parts, int k, int ldz,
                                                                         int tiles_m, int tiles_n, int group_m, int band, ColumnsEnd end) {
    __shared__ __attribute__((aligned(1024))) char lds[RingLds<BM, BN, WGM, WGN, WGK>::BYTES];
    gemm_ring_tile<BM, BN, WGM, WGN, WGK, false, false, EPI_OWN, true>(lds, (const bf16_t*)h, (const bf16_t*)parts, nullptr, nullptr, nullptr, nullptr, end.m, ldz, k,
                                                                       end.m, ldz, EPI_OWN, 0, 0, tiles_m, tiles_n, group_m, (int)blockIdx.x, nullptr, true, 0,
                                                                       Ahead{nullptr, 0}, band, end);
}

// ---- float: a piece of z is in memory, [m, ld], of which `cols` columns from v0 on count
__global__ __launch_bounds__(ROW_THREADS) void xent_stats_f32_kernel(const float* __restrict__ z, int ld, int cols, int v0, int vocab, const int* __restrict__ targets,
                                                                     float2* __restrict__ stats, float* __restrict__ at_target) {
    __shared__ float2 part[ROW_THREADS / WAVE];
    const int t = blockIdx.x, tid = threadIdx.x;
    const float* row = z + (size_t)t * ld;
    float2 s = make_float2(LOWEST, 0.f);
    for (int c = tid * 4; c < cols; c += ROW_THREADS * 4) {
        float v[4];
        load_vec<float>(row + c, v);
        float top = LOWEST, sum = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (c + e >= cols) v[e] = -INFINITY;
            top = fmaxf(top, v[e]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) sum += __builtin_amdgcn_exp2f((v[e] - top) * LOG2E);
        s = join(s, make_float2(top, sum));
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
__global__ __launch_bounds__(ROW_THREADS) void xent_dz_f32_kernel(float* __restrict__ z, int ld, int cols, int v0, int vocab, const int* __restrict__ targets,
                                                                  const float* __restrict__ lse, const float* __restrict__ dloss, float scale) {
    const int t = blockIdx.x, target = targets[t];
    const float coef = counts(target, vocab) ? (dloss ? scale * dloss[t] : scale) : 0.f, l = lse[t];
    float* row = z + (size_t)t * ld;
    for (int c = threadIdx.x * 4; c < ld; c += ROW_THREADS * 4) {
        float v[4];
        load_vec<float>(row + c, v);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float d = __builtin_amdgcn_exp2f((v[e] - l) * LOG2E) - (c + e == target - v0 ? 1.0f : 0.0f);
            v[e] = coef == 0.f || c + e >= cols ? 0.f : coef * d;
        }
        store_vec<float>(row + c, v);
    }
}
// columns of a wider matrix: to (+)= from [rows, ld], `cols` of them
__global__ __launch_bounds__(ROW_THREADS) void xent_columns_kernel(const float* __restrict__ from, int ld, int cols, float* __restrict__ to, int ldto, int overwrite) {
    const int c = (blockIdx.x * ROW_THREADS + threadIdx.x) * 4;
    if (c >= cols) return;
    float v[4], o[4] = {0.f, 0.f, 0.f, 0.f};
    load_vec<float>(from + (size_t)blockIdx.y * ld + c, v);
    float* dst = to + (size_t)blockIdx.y * ldto + c;
    if (!overwrite) load_vec<float>(dst, o);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] += o[e];
    if (c + 4 <= cols) store_vec<float>(dst, v);
    else
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (c + e < cols) dst[e] = v[e];
}

size_t aligned(size_t b) { return (b + 255) / 256 * 256; }
int round_up(int v, int a) { return (v + a - 1) / a * a; }
long tiles_of(int m, int n, int tile) { return (long)((m + tile - 1) / tile) * ((n + tile - 1) / tile); }
double rounds(long tiles) { return (double)((tiles + NUM_CUS - 1) / NUM_CUS); }

// 256x256 tiles where they fill most of the chip, else 128x128 (as for the stages' products).
int z_tile(int m, int n) { return tiles_of(m, n, 256) >= 144 ? 256 : 128; }

// Columns of the vocabulary per piece where the caller leaves it open: dz of a piece takes at most this.
constexpr size_t PIECE_BYTES = (size_t)512 << 20;
constexpr int PIECE_STEP = 256;
// Time of a round of tiles per step of 64 of the contraction, us (one tile per CU; see split_plan in gemm_mfma.hip)
constexpr double STEP256 = 1.4, STEP128 = 0.5, SLAB = 8 / 4.5e6, LAUNCH = 10;
double product_cost(int m, int n, long k) {
    const double steps = (double)((k + 63) / 64);
    return z_tile(m, n) == 256 ? rounds(tiles_of(m, n, 256)) * steps * STEP256 : rounds(tiles_of(m, n, 128)) * steps * STEP128;
}
struct SplitOf { int tile, splits, k_per; double cost; };
// How the contraction of dh over a piece is cut: slabs are read and written once for every piece.
SplitOf split_of(int m, int n, int k) {
    const long steps = (k + 63) / 64;
    SplitOf best{256, 1, round_up(k, 64), 1e300};
    for (int tile : {256, 128})
        for (int s = 1; s <= 64 && (s == 1 || steps / s >= 4); ++s) {
            const long per = (steps + s - 1) / s;
            if ((steps + per - 1) / per != s) continue;
            const double cost = rounds(tiles_of(m, n, tile) * s) * per * (tile == 256 ? STEP256 : STEP128) + SLAB * s * m * n;
            if (cost < best.cost) best = {tile, s, (int)per * 64, cost};
        }
    return best;
}
int default_piece(int dtype, int m, int hidden, int vocab) {
    const int all = round_up(vocab, PIECE_STEP), mp = round_up(m, TOKEN_PAD);
    const size_t column = dtype == CHIMERA_F32 ? ((size_t)m + hidden) * 4 : (size_t)mp * 6;
    const int most = std::max<int>(PIECE_STEP, (int)std::min<size_t>(all, PIECE_BYTES / column / PIECE_STEP * PIECE_STEP));
    if (most >= all) return all;
    int best = most;
    double least = 1e300;
    for (int p = most; p >= PIECE_STEP && p >= most / 2; p -= PIECE_STEP) {
        const int n = (vocab + p - 1) / p;
        const double cost = n * (product_cost(m, p, hidden) + product_cost(hidden, p, 2l * mp) + split_of(m, hidden, p).cost + 3 * LAUNCH);
        if (cost < least) { least = cost; best = p; }
    }
    return best;
}

struct FwdLayout { int tile, parts; size_t stats, at_target, z, total; int piece; };
FwdLayout fwd_layout(int dtype, int m, int hidden, int vocab) {
    FwdLayout l{};
    size_t b = 0;
    auto take = [&](size_t bytes) { size_t r = b; b += aligned(bytes); return r; };
    l.tile = z_tile(m, vocab);
    l.piece = default_piece(dtype, m, hidden, vocab);
    l.parts = dtype == CHIMERA_F32 ? (vocab + l.piece - 1) / l.piece : (vocab + l.tile - 1) / l.tile;
    l.stats = take((size_t)l.parts * m * sizeof(float2));
    l.at_target = take((size_t)m * 4);
    l.z = take(dtype == CHIMERA_F32 ? (size_t)m * std::min(l.piece, round_up(vocab, 8)) * 4 : 0);
    l.total = b;
    return l;
}
struct BwdLayout { int piece, ld, mp; SplitOf split; size_t rows, up, room, shift, dz, parts, slabs, columns, total; };
BwdLayout bwd_layout(int dtype, int m, int hidden, int vocab, int piece) {
    BwdLayout l{};
    size_t b = 0;
    auto take = [&](size_t bytes) { size_t r = b; b += aligned(bytes); return r; };
    const bool f32 = dtype == CHIMERA_F32;
    l.piece = piece ? round_up(piece, PIECE_STEP) : default_piece(dtype, m, hidden, vocab);
    l.ld = std::min(l.piece, round_up(vocab, 8));
    l.mp = f32 ? m : round_up(m, TOKEN_PAD);
    l.split = f32 ? SplitOf{0, 1, l.ld, 0} : split_of(m, hidden, l.ld);
    l.rows = take((size_t)l.mp * hidden * 4);                       // float rows, or fp16 rows twice
    l.up = take((size_t)m * 4);
    l.room = take((size_t)m * 4);
    l.shift = take(4);
    l.dz = take((size_t)l.mp * l.ld * (f32 ? 4 : 2));
    l.parts = take(f32 ? 0 : (size_t)l.mp * l.ld * 4);
    l.slabs = take((size_t)l.split.splits * m * hidden * 4);
    l.columns = take(f32 ? (size_t)hidden * l.ld * 4 : 0);
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
    if (tokens > 1 << 22 || hidden > 1 << 16 || vocab > 1 << 22) return fail(CHIMERA_EINVAL, "more than 2^22 tokens, 2^16 hidden or 2^22 vocabulary columns");
    if (hidden % 8) return fail(CHIMERA_EINVAL, "hidden=%d must be a multiple of 8", hidden);
    if (ldh % 8 || ldw % 8) return fail(CHIMERA_EINVAL, "leading dimensions ldh=%d, ldw=%d must be multiples of 8", ldh, ldw);
    if (ldh < hidden || ldw < vocab) return fail(CHIMERA_EINVAL, "leading dimension too small");
    if (ldh >= 1 << 23 || ldw >= 1 << 23) return fail(CHIMERA_EINVAL, "leading dimension of 2^23 or more");
    return CHIMERA_OK;
}

template <int BM, int WGM, int WGN, int WGK, typename F>
int with_raster(int m, int n, int k, F&& launch) {
    const int tm = (m + BM - 1) / BM, tn = (n + BM - 1) / BM;
    constexpr int PER_CU = RingLds<BM, BM, WGM, WGN, WGK>::PER_CU;
    const int band = raster_band(tm, tn, NUM_CUS * PER_CU, (size_t)n * k * 2);
    const int gm = raster_group(tm, band ? band : tn, std::min((tm * tn + 7) / 8, PER_XCD * PER_CU), BM, BM);
    launch(tm, tn, gm, band);
    CHIMERA_LAUNCH_CHECK("linear cross-entropy");
    return CHIMERA_OK;
}
// The launches of a product m x n on one of the three forms of tiles: f.operator()<BM, WGM, WGN, WGK>()
template <typename F> int with_tile(int m, int n, F&& f) {
    if (z_tile(m, n) == 256) return f.template operator()<256, 2, 4, 1>();
    if (tiles_of(m, n, 128) <= NUM_CUS) return f.template operator()<128, 2, 2, 2>();
    return f.template operator()<128, 2, 2, 1>();
}

int xent_fwd_f32(int m, int hidden, int vocab, const float* h, int ldh, const float* w, int ldw, const int* targets, const FwdLayout& l, char* ws, void* stream) {
    for (int v0 = 0, p = 0; v0 < vocab; v0 += l.piece, ++p) {
        const int cols = std::min(l.piece, vocab - v0), ld = round_up(cols, 8);
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
    float *rows = (float*)(ws + l.rows), *z = (float*)(ws + l.dz), *slab = (float*)(ws + l.slabs), *columns = (float*)(ws + l.columns);
    if (dw) {
        hipLaunchKernelGGL((xent_rows_kernel<float, float>), dim3((m + 3) / 4), dim3(ROW_THREADS), 0, s, h, ldh, targets, dloss, scale, m, m, hidden, vocab, rows,
                           nullptr, nullptr);
        CHIMERA_LAUNCH_CHECK("linear cross-entropy");
    }
    int slabs = 0;
    for (int v0 = 0; v0 < vocab; v0 += l.piece) {
        const int cols = std::min(l.piece, vocab - v0), ld = round_up(cols, 8), whole = cols & ~7;
        GemmArgs g{};
        g.m = m; g.n = ld; g.k = hidden; g.a = h; g.lda = ldh; g.a_kc = 1; g.b = w + v0; g.ldb = ldw; g.b_kc = 0; g.c = z; g.epilogue = EPI_NONE;
        XENT_TRY(gemm_f32(g, stream));
        hipLaunchKernelGGL(xent_dz_f32_kernel, dim3(m), dim3(ROW_THREADS), 0, s, z, ld, cols, v0, vocab, targets, lse, dloss, scale);
        CHIMERA_LAUNCH_CHECK("linear cross-entropy");
        if (dh && whole) {
            GemmArgs d{};
            d.m = m; d.n = hidden; d.k = whole; d.a = z; d.lda = ld; d.a_kc = 1; d.b = w + v0; d.ldb = ldw; d.b_kc = 1; d.c = slab;
            d.epilogue = slabs ? EPI_ACCUM_F32 : EPI_NONE;
            XENT_TRY(gemm_f32(d, stream));
            slabs = 1;
        }
        if (dw) {
            GemmArgs q{};
            q.m = hidden; q.n = ld; q.k = m; q.a = rows; q.lda = hidden; q.a_kc = 0; q.b = z; q.ldb = ld; q.b_kc = 0; q.c = columns; q.epilogue = EPI_ACCUM_F32;
            XENT_TRY(gemm_f32_group(1, &q, nullptr, 1, stream));
            hipLaunchKernelGGL(xent_columns_kernel, dim3((cols + ROW_THREADS * 4 - 1) / (ROW_THREADS * 4), hidden), dim3(ROW_THREADS), 0, s, columns, ld, cols,
                               dw + v0, lddw, overwrite);
            CHIMERA_LAUNCH_CHECK("linear cross-entropy");
        }
        if (dh && v0 + l.piece >= vocab) {
            hipLaunchKernelGGL(xent_dh_sum_kernel<float>, dim3((m + DH_ROWS - 1) / DH_ROWS, (hidden / 4 + ROW_THREADS - 1) / ROW_THREADS), dim3(ROW_THREADS), 0, s,
                               slab, slabs, z + whole, ld, w + v0 + whole, ldw, cols - whole, m, hidden, dh, lddh);
            CHIMERA_LAUNCH_CHECK("linear cross-entropy");
        }
    }
    return CHIMERA_OK;
}

int xent_bwd_bf16(int m, int hidden, int vocab, const bf16_t* h, int ldh, const bf16_t* w, int ldw, const int* targets, const float* lse, float scale,
                  const float* dloss, bf16_t* dh, int lddh, float* dw, int lddw, int overwrite, const BwdLayout& l, char* ws, void* stream) {
    hipStream_t s = (hipStream_t)stream;
    _Float16 *rows = (_Float16*)(ws + l.rows), *parts = (_Float16*)(ws + l.parts);
    int *up = (int*)(ws + l.up), *room = (int*)(ws + l.room), *shift = (int*)(ws + l.shift);
    bf16_t* dz = (bf16_t*)(ws + l.dz);
    float* slabs = (float*)(ws + l.slabs);
    hipLaunchKernelGGL((xent_rows_kernel<bf16_t, _Float16>), dim3((l.mp + 3) / 4), dim3(ROW_THREADS), 0, s, h, ldh, targets, dloss, scale, m, l.mp, hidden, vocab,
                       rows, up, room);
    CHIMERA_LAUNCH_CHECK("linear cross-entropy");
    hipLaunchKernelGGL(xent_shift_kernel, dim3(1), dim3(1024), 0, s, room, m, shift);
    CHIMERA_LAUNCH_CHECK("linear cross-entropy");
    int splits = 0;
    for (int v0 = 0; v0 < vocab; v0 += l.piece) {
        const int cols = std::min(l.piece, vocab - v0), ld = round_up(cols, 8), whole = cols & ~7;
        XENT_TRY(with_tile(m, ld, [&]<int BM, int WGM, int WGN, int WGK>() {
            return with_raster<BM, WGM, WGN, WGK>(l.mp, ld, hidden, [&](int tm, int tn, int gm, int band) {
                const GradEnd<BM, WGM * WGN * WGK> end{lse, targets, dloss, up, shift, scale, m, l.mp, vocab, v0, cols, ld, dz, parts, {}};
                hipLaunchKernelGGL((xent_dz_kernel<BM, BM, WGM, WGN, WGK>), dim3(tm * tn), dim3(WGM * WGN * WGK * 64), 0, s, h, w, hidden, ldh, ldw, tm, tn, gm,
                                   band, end);
            });
        }));
        if (dh && whole) {
            // the last piece is cut where the others are: a split that it does not reach adds nothing
            const int t = l.split.tile, tm = (m + t - 1) / t, tn = (hidden + t - 1) / t, now = (whole + l.split.k_per - 1) / l.split.k_per;
            const int gm = raster_group(tm, tn, std::min(tm * tn, (tm * tn * now + 7) / 8), t, t);
            const dim3 grid(tm * tn * now), block(512);
            const int flags = splits ? 0 : ACCUM_OVERWRITE;
#define XENT_DH(...) hipLaunchKernelGGL((xent_dh_kernel<__VA_ARGS__>), grid, block, 0, s, dz, w + v0, slabs, m, hidden, whole, ld, ldw, tm, tn, gm, now, l.split.k_per, flags)
            if (t == 256) XENT_DH(256, 256, 2, 4, 1);
            else XENT_DH(128, 128, 2, 2, 2);
#undef XENT_DH
            CHIMERA_LAUNCH_CHECK("linear cross-entropy");
            if (!splits) splits = now;
        }
        if (dw)
            XENT_TRY(with_tile(hidden, ld, [&]<int BM, int WGM, int WGN, int WGK>() {
                return with_raster<BM, WGM, WGN, WGK>(hidden, ld, 2 * l.mp, [&](int tm, int tn, int gm, int band) {
                    const ColumnsEnd end{dw + v0, shift, hidden, cols, lddw, overwrite ? ACCUM_OVERWRITE : 0};
                    hipLaunchKernelGGL((xent_dw_kernel<BM, BM, WGM, WGN, WGK>), dim3(tm * tn), dim3(WGM * WGN * WGK * 64), 0, s, rows, parts, 2 * l.mp, ld, tm, tn,
                                       gm, band, end);
                });
            }));
        if (dh && v0 + l.piece >= vocab) {
            hipLaunchKernelGGL(xent_dh_sum_kernel<bf16_t>, dim3((m + DH_ROWS - 1) / DH_ROWS, (hidden / 4 + ROW_THREADS - 1) / ROW_THREADS), dim3(ROW_THREADS), 0, s,
                               slabs, splits, dz + whole, ld, w + v0 + whole, ldw, cols - whole, m, hidden, dh, lddh);
            CHIMERA_LAUNCH_CHECK("linear cross-entropy");
        }
    }
    return CHIMERA_OK;
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
    char* ws = (char*)d_workspace;
    float2* stats = (float2*)(ws + l.stats);
    float* at_target = (float*)(ws + l.at_target);
    hipStream_t s = (hipStream_t)hip_stream;
    if (dtype == CHIMERA_F32)
        XENT_TRY(xent_fwd_f32(tokens, hidden, vocab, (const float*)d_h, ldh, (const float*)d_w, ldw, d_targets, l, ws, hip_stream));
    else
        XENT_TRY(with_tile(tokens, vocab, [&]<int BM, int WGM, int WGN, int WGK>() {
            return with_raster<BM, WGM, WGN, WGK>(tokens, vocab, hidden, [&](int tm, int tn, int gm, int band) {
                hipLaunchKernelGGL((xent_stats_kernel<BM, BM, WGM, WGN, WGK>), dim3(tm * tn), dim3(WGM * WGN * WGK * 64), 0, s, (const bf16_t*)d_h,
                                   (const bf16_t*)d_w, d_targets, stats, at_target, tokens, vocab, hidden, ldh, ldw, tm, tn, gm, band);
            });
        }));
    hipLaunchKernelGGL(xent_join_kernel, dim3((tokens + 15) / 16), dim3(256), 0, s, stats, at_target, d_targets, tokens, vocab, l.parts, scale, d_loss_rows, d_lse);
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
