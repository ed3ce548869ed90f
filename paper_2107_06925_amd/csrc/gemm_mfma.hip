// bf16 GEMM on the CDNA4 matrix cores, float accumulation, for the three products of a linear layer:
//   forward  Y  = X W      A k-contiguous, B stored [k, n]
//   dgrad    dX = dY W^T   A k-contiguous, B k-contiguous
//   wgrad    dW += X^T dY  A stored [k, m], B stored [k, n]  (k = tokens)
//
// One workgroup computes a tile of the output; its wavefronts own parts of it as a grid of MFMA
// tiles whose accumulators never leave the registers.  Three kernels, by size (choose_tile):
//   gemm_ring_tile    256x256, 256x128 and 128x128 tiles on v_mfma_f32_16x16x32_bf16
//   gemm_async_tile   32x32 to 128x64 tiles on v_mfma_f32_32x32x16_bf16, a ring of k steps
//   gemm_bf16_kernel  the register-staged form: split-K and shapes on request
// The k loop moves BK = 64 at a time through LDS, the next steps in flight.  What follows on
// LDS layouts is the latter two's; gemm_ring_tile's own differ in their exchanges and are described there.
//
// An operand that is k-contiguous in memory (X in the forward, both operands of
// dgrad) sits in LDS as [row][k], 128 bytes per row, and lane l reads its MFMA
// operand - row l%32, the 8 consecutive k of chunk 2*kk + l/32 - with one
// 16-byte load.  Chunk c of row r is stored at c ^ (r & 7) ^ ((r >> 3) & 7), so the
// 8 rows a read touches per bank cycle fall on 8 different bank groups.
// An operand whose OTHER index is contiguous in memory (W in the forward, both
// operands of wgrad) is copied to LDS as it lies in memory, [k][row], and the
// transposition is done by the LDS hardware: ds_read_b64_tr_b16 hands lane i of
// each 16-lane group the i-th 16-bit element of the data addressed by lanes
// 4e + i/4 (e = 0..3), i.e. column i of a 4 x 16 block - four consecutive k of one
// row.  Two such reads give the same 8 k values the other flavour gets from one
// 16-byte load.  The 32-byte column blocks of row k are stored at block ^ 2(k & 3):
// one bank cycle serves 32 lanes = two adjacent column blocks x four rows, and this
// puts those eight 32-byte pieces on eight different bank groups (measured: without
// it half of the LDS cycles of the wgrad kernel were bank conflicts).  No transposed
// copy of any activation or weight exists in HBM, and no data is shuffled in
// registers.
//
// Workgroups are renumbered so that each of the 8 XCDs (own L2 each; the
// hardware deals consecutive workgroup ids round-robin over them) works on a
// contiguous range of tiles, and tiles are walked in groups of 8 tile rows so
// that the tiles in flight on one XCD share operand panels in its L2.
#include "gemm_tiles.h"

#include <algorithm>
#include <climits>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <type_traits>

namespace chimera {

namespace {

template <int BM, int BN, int WGM, int WGN, int PF, bool A_KC, bool B_KC>
__global__ __launch_bounds__(WGM* WGN * 64) void gemm_bf16_kernel(
    const bf16_t* __restrict__ A, const bf16_t* __restrict__ B, const bf16_t* __restrict__ bias,
    const bf16_t* __restrict__ R, void* __restrict__ C, bf16_t* __restrict__ C2, int m, int n, int k, int lda,
    int ldb, int epi, int epi_flag, int res_types, int tiles_m, int tiles_n, int splits, float* __restrict__ slabs,
    unsigned* __restrict__ arrivals) {
    constexpr int NT = WGM * WGN * 64;
    constexpr int WM = BM / WGM, WN = BN / WGN;    // wavefront tile
    constexpr int TM = WM / 32, TN = WN / 32;      // MFMA tiles per wavefront
    __shared__ __attribute__((aligned(16))) bf16_t lds[2][(BM + BN) * BK];

    // workgroup id -> tile, XCD-contiguous then grouped raster
    // With split-K the grid holds `splits` workgroups per tile: split = blockIdx / tiles.
    const int nblk = tiles_m * tiles_n;
    const int split = blockIdx.x / nblk, bid = blockIdx.x % nblk;
    const int xcd = bid & 7, local = bid >> 3;
    const int pid = xcd * (nblk >> 3) + min(xcd, nblk & 7) + local;
    const int width = GROUP_M * tiles_n;
    const int first_m = (pid / width) * GROUP_M;
    const int gsz = min(tiles_m - first_m, GROUP_M);
    const int tile_m = first_m + (pid % width) % gsz;
    const int tile_n = (pid % width) / gsz;
    const int i0 = tile_m * BM, j0 = tile_n * BN;

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int wm0 = (wave / WGN) * WM, wn0 = (wave % WGN) * WN;

    f32x16 acc[TM][TN];
#pragma unroll
    for (int a = 0; a < TM; ++a)
#pragma unroll
        for (int b = 0; b < TN; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[a][b][r] = 0.f;

    // one k step of MFMA work out of LDS buffer `buf`
    auto compute = [&](int buf) {
        const bf16_t* As = lds[buf];
        const bf16_t* Bs = lds[buf] + BM * BK;
#pragma unroll
        for (int kk = 0; kk < BK / 16; ++kk) {
            bf16x8 af[TM], bfr[TN];
#pragma unroll
            for (int a = 0; a < TM; ++a) af[a] = read_frag<BM, A_KC>(As, wm0 + a * 32, kk, lane);
#pragma unroll
            for (int b = 0; b < TN; ++b) bfr[b] = read_frag<BN, B_KC>(Bs, wn0 + b * 32, kk, lane);
#pragma unroll
            for (int a = 0; a < TM; ++a)
#pragma unroll
                for (int b = 0; b < TN; ++b)
                    acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bfr[b], af[a], acc[a][b], 0, 0, 0);
        }
    };
    auto fetch = [&](Staged<BM, NT, A_KC>& ra, Staged<BN, NT, B_KC>& rb, int kt) {
        load_tile<BM, NT, A_KC>(ra, A, lda, i0, m, kt * BK, k, tid);
        load_tile<BN, NT, B_KC>(rb, B, ldb, j0, n, kt * BK, k, tid);
    };
    auto stash = [&](const Staged<BM, NT, A_KC>& ra, const Staged<BN, NT, B_KC>& rb, int buf) {
        store_tile<BM, NT, A_KC>(ra, lds[buf], tid);
        store_tile<BN, NT, B_KC>(rb, lds[buf] + BM * BK, tid);
    };

    // Software pipeline: global loads run PF k steps ahead of the matrix cores in PF
    // register sets (a ring walked by an unrolled loop, so every index is static),
    // LDS runs one step ahead in two buffers, one barrier per step.
    // This workgroup's share of the k steps: [K0, K1).
    const int KT_all = (k + BK - 1) / BK;
    const int K0 = (int)((long)KT_all * split / splits), K1 = (int)((long)KT_all * (split + 1) / splits);
    const int KT = K1 - K0;
    Staged<BM, NT, A_KC> ra[PF];
    Staged<BN, NT, B_KC> rb[PF];
#pragma unroll
    for (int u = 0; u < PF; ++u)
        if (u < KT) fetch(ra[u], rb[u], K0 + u);
    stash(ra[0], rb[0], 0);
    __syncthreads();
    for (int kt = 0; kt < KT; kt += PF) {
#pragma unroll
        for (int u = 0; u < PF; ++u) {
            const int step = kt + u;
            if (step >= KT) break;
            if (step + PF < KT) fetch(ra[u], rb[u], K0 + step + PF);      // set u was stashed one step ago
            compute(step & 1);
            if (step + 1 < KT) stash(ra[(u + 1) % PF], rb[(u + 1) % PF], (step + 1) & 1);
            __syncthreads();
        }
    }

    // Split-K: every workgroup of a tile writes its partial accumulators to its own slab
    // (thread-private order, 16-byte stores), then counts itself in.  Whoever arrives last
    // adds the slabs in split order - so the sum does not depend on who that is - and runs
    // the epilogue.  Nobody waits for anybody.
    if (splits > 1) {
        __shared__ int is_last;
        const size_t tile_elems = (size_t)BM * BN;
        float4* mine = reinterpret_cast<float4*>(slabs + ((size_t)split * nblk + pid) * tile_elems);
#pragma unroll
        for (int a = 0; a < TM; ++a)
#pragma unroll
            for (int b = 0; b < TN; ++b)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    mine[((a * TN + b) * 4 + q) * NT + tid] =
                        make_float4(acc[a][b][4 * q], acc[a][b][4 * q + 1], acc[a][b][4 * q + 2], acc[a][b][4 * q + 3]);
        __threadfence();                       // slab visible device-wide before the arrival count
        __syncthreads();
        if (tid == 0) is_last = atomicAdd(&arrivals[pid], 1u) == (unsigned)(splits - 1);
        __syncthreads();
        if (!is_last) return;
        __threadfence();                       // see the other workgroups' slabs
#pragma unroll
        for (int a = 0; a < TM; ++a)
#pragma unroll
            for (int b = 0; b < TN; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[a][b][r] = 0.f;
        for (int sp = 0; sp < splits; ++sp) {
            const float4* other = reinterpret_cast<const float4*>(slabs + ((size_t)sp * nblk + pid) * tile_elems);
#pragma unroll
            for (int a = 0; a < TM; ++a)
#pragma unroll
                for (int b = 0; b < TN; ++b)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const float4 v = other[((a * TN + b) * 4 + q) * NT + tid];
                        acc[a][b][4 * q] += v.x; acc[a][b][4 * q + 1] += v.y;
                        acc[a][b][4 * q + 2] += v.z; acc[a][b][4 * q + 3] += v.w;
                    }
        }
        if (tid == 0) arrivals[pid] = 0u;      // ready for the next launch on this stream
    }

    const int rb0 = i0 + wm0, cb0 = j0 + wn0;
    // the operand tiles in LDS are dead once every wavefront has left the k loop; each
    // wavefront then stages its output through its own slab there
    static_assert(sizeof(lds) >= (size_t)WGM * WGN * EpiSlab<TN>::FLOATS * sizeof(float), "LDS too small for the epilogue");
    __syncthreads();
    float* slab = reinterpret_cast<float*>(lds) + (size_t)(tid >> 6) * EpiSlab<TN>::FLOATS;
    with_epilogue(epi, res_types, [&]<int E, bool RF, bool CF>() {
        epilogue<E, RF, CF, TM, TN>(Acc32<TM, TN>{acc}, slab, rb0, cb0, m, n, bias, R, C, C2, epi_flag, lane);
    });
}

template <int BM, int BN, int WGM, int WGN, int WGK, bool A_KC, bool B_KC>
__global__ __launch_bounds__(WGM* WGN * WGK * 64, 2) void gemm_bf16_ring_kernel(
    const bf16_t* __restrict__ A, const bf16_t* __restrict__ B, const bf16_t* __restrict__ bias,
    const bf16_t* __restrict__ R, void* __restrict__ C, bf16_t* __restrict__ C2, int m, int n, int k, int lda,
    int ldb, int epi, int epi_flag, int res_types, int tiles_m, int tiles_n, int group_m, int band, int col0, Ahead ahead) {
    __shared__ __attribute__((aligned(1024))) char lds[RingLds<BM, BN, WGM, WGN, WGK>::BYTES];
    gemm_ring_tile<BM, BN, WGM, WGN, WGK, A_KC, B_KC, -1>(lds, A, B, bias, R, C, C2, m, n, k, lda, ldb, epi, epi_flag, res_types,
                                                          tiles_m, tiles_n, group_m, (int)blockIdx.x, nullptr, true, col0, ahead, band);
}

// A long contraction with few output tiles, cut along k: workgroups [s * tiles, (s+1) * tiles) (numbered so
// that an XCD works on few splits) write the partial sums over k in [s * k_per, (s+1) * k_per) to float slab s;
// split_sum_kernel adds the slabs in their order.  No workgroup waits for another.
template <int BM, int BN, int WGM, int WGN, int WGK>
__global__ __launch_bounds__(WGM* WGN * WGK * 64, 2) void gemm_bf16_ring_split_kernel(
    const bf16_t* __restrict__ A, const bf16_t* __restrict__ B, float* __restrict__ slabs, int m, int n, int k, int lda, int ldb,
    int tiles_m, int tiles_n, int group_m, int splits, int k_per) {
    const int tiles = tiles_m * tiles_n, total = tiles * splits;
    const int xcd = (int)blockIdx.x & 7, local = (int)blockIdx.x >> 3;
    const int pid = xcd * (total >> 3) + min(xcd, total & 7) + local;
    const int split = pid / tiles, k0 = split * k_per;
    __shared__ __attribute__((aligned(1024))) char lds[RingLds<BM, BN, WGM, WGN, WGK>::BYTES];
    gemm_ring_tile<BM, BN, WGM, WGN, WGK, true, true, EPI_ACCUM_F32>(
        lds, A + k0, B + k0, nullptr, nullptr, slabs + (size_t)split * m * n, nullptr, m, n, min(k_per, k - k0), lda, ldb,
        EPI_ACCUM_F32, 1, 0, tiles_m, tiles_n, group_m, pid % tiles, nullptr, false);
}

__global__ __launch_bounds__(256) void split_sum_kernel(const float* __restrict__ slabs, size_t elems, int splits, bf16_t* __restrict__ c) {
    const size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (i >= elems) return;
    float v[8];
    load8(slabs + i, v);
    for (int s = 1; s < splits; ++s) {
        float u[8];
        load8(slabs + (size_t)s * elems + i, u);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += u[e];
    }
    store8(c + i, v);
}

template <int BM, int BN, int WGM, int WGN, int WGK, int NS, int SPS, bool A_KC, bool B_KC>
__global__ __launch_bounds__(WGM* WGN * WGK * 64) void gemm_bf16_async_kernel(
    const bf16_t* __restrict__ A, const bf16_t* __restrict__ B, const bf16_t* __restrict__ bias,
    const bf16_t* __restrict__ R, void* __restrict__ C, bf16_t* __restrict__ C2, int m, int n, int k, int lda,
    int ldb, int epi, int epi_flag, int res_types, int tiles_m, int tiles_n, int group_m, Ahead ahead) {
    gemm_async_tile<BM, BN, WGM, WGN, WGK, NS, SPS, A_KC, B_KC, -1>(A, B, bias, R, C, C2, m, n, k, lda, ldb, epi, epi_flag,
                                                                res_types, tiles_m, tiles_n, group_m, (int)blockIdx.x, nullptr,
                                                                true, ahead);
}

// Several products C_p (float) += A_p B_p of one launch: same contraction length and operand
// layout, each with its own shapes and pointers.  Workgroups [first[p], first[p+1]) work on
// product p, so small products no longer leave most of the chip idle for a launch of their
// own.  (The weight gradients of one Transformer block are such a group.)
constexpr int GROUP_MAX = 4;
struct GemmGroup {
    const bf16_t* a[GROUP_MAX];
    const bf16_t* b[GROUP_MAX];
    float* c[GROUP_MAX];
    float* bsum[GROUP_MAX];      // optional: bsum[j] += sum_k B(k, j)
    int m[GROUP_MAX], n[GROUP_MAX], lda[GROUP_MAX], ldb[GROUP_MAX], tiles_m[GROUP_MAX], tiles_n[GROUP_MAX];
    int group_m[GROUP_MAX];      // tile rows per raster group of each product
    int first[GROUP_MAX + 1];
    int count, k;
    int overwrite;               // results replace C and bsum instead of being added
};

// The product of a group launch that this workgroup belongs to, and its tile's number inside the
// group: each XCD takes a contiguous range of the group's tiles (products laid end to end), so that
// its L2 sees few operand panels: one product's tiles are not dealt over all eight XCDs.
__device__ __forceinline__ int group_product(const GemmGroup& grp, int& gid) {
    const int total = grp.first[grp.count];
    const int xcd = (int)blockIdx.x & 7, local = (int)blockIdx.x >> 3;
    gid = xcd * (total >> 3) + min(xcd, total & 7) + local;
    int p = 0;
#pragma unroll
    for (int i = 1; i < GROUP_MAX; ++i)
        if (i < grp.count && gid >= grp.first[i]) p = i;
    return p;
}

template <int BM, int BN, int WGM, int WGN, int WGK>
__global__ __launch_bounds__(WGM* WGN * WGK * 64, 2) void gemm_bf16_ring_group_kernel(GemmGroup grp) {
    int gid;
    const int p = group_product(grp, gid);
    __shared__ __attribute__((aligned(1024))) char lds[RingLds<BM, BN, WGM, WGN, WGK>::BYTES];
    gemm_ring_tile<BM, BN, WGM, WGN, WGK, false, false, EPI_ACCUM_F32>(
        lds, grp.a[p], grp.b[p], nullptr, nullptr, grp.c[p], nullptr, grp.m[p], grp.n[p], grp.k, grp.lda[p], grp.ldb[p],
        EPI_ACCUM_F32, grp.overwrite, 0, grp.tiles_m[p], grp.tiles_n[p], grp.group_m[p], gid - grp.first[p], grp.bsum[p],
        false);
}

template <int BM, int BN, int WGM, int WGN, int WGK, int NS, int SPS, bool A_KC, bool B_KC>
__global__ __launch_bounds__(WGM* WGN * WGK * 64) void gemm_bf16_async_group_kernel(GemmGroup grp) {
    int gid;
    const int p = group_product(grp, gid);
    gemm_async_tile<BM, BN, WGM, WGN, WGK, NS, SPS, A_KC, B_KC, EPI_ACCUM_F32>(
        grp.a[p], grp.b[p], nullptr, nullptr, grp.c[p], nullptr, grp.m[p], grp.n[p], grp.k, grp.lda[p], grp.ldb[p],
        EPI_ACCUM_F32, grp.overwrite, 0, grp.tiles_m[p], grp.tiles_n[p], grp.group_m[p], gid - grp.first[p], grp.bsum[p],
        false);
}

// The same on tiles of several sizes in one launch.  An entry is the tiles of one size of one product, a phase the entries of all products
// that are begun together.  Of every 256 tiles of a phase an XCD takes 32 neighbours, so that the tiles in flight share operand panels in
// its L2 and, between the XCDs, in the memory-side cache (one range of the whole phase per XCD: block of 2048 at k = 512 121 -> 128 us, of
// 1920 at 2048 204 -> 220; one range of each product's tiles: block of 1280 at 2048 104 -> 128).
enum TileForm { TILE_256, TILE_128x256, TILE_256x128, TILE_128 };
constexpr int MIXED_MAX = 5 * GROUP_MAX;
struct MixedEntry {
    const bf16_t *a, *b;
    float *c, *bsum;
    int m, n, lda, ldb, tiles_m, tiles_n, group_m, band, col0;
    int form;
};
constexpr int MIXED_PHASES = 3;
struct MixedPhase {
    int first, tiles;                // its tiles
    int local;                       // number, within an XCD, of its first workgroup
    int skew;                        // the XCD that takes the first of the tiles that eight do not divide
};
struct MixedGroup {
    MixedPhase phase[MIXED_PHASES];
    int first[MIXED_MAX];            // number of an entry's first tile, all laid end to end (INT_MAX behind the last entry)
    int count, k, flags;             // flags: ACCUM_*
    MixedEntry e[MIXED_MAX];
};

__global__ __launch_bounds__(512, 2) void gemm_bf16_mixed_group_kernel(MixedGroup grp) {
    __shared__ __attribute__((aligned(1024))) char lds[RingLds<256, 128, 2, 2, 2>::BYTES];
    static_assert(RingLds<256, 256, 2, 4, 1>::BYTES <= sizeof(lds) && RingLds<128, 256, 1, 4, 2>::BYTES <= sizeof(lds) &&
                  RingLds<128, 128, 2, 2, 2>::BYTES <= sizeof(lds), "the largest of them");
    const int local = (int)blockIdx.x >> 3, h = local >= grp.phase[2].local ? 2 : local >= grp.phase[1].local ? 1 : 0;
    const MixedPhase& p = grp.phase[h];
    const int slot = ((int)blockIdx.x - p.skew) & 7, at = local - p.local, rounds = p.tiles / NUM_CUS, rest = p.tiles % NUM_CUS;
    int gid = p.first + at / PER_XCD * NUM_CUS + slot * PER_XCD + at % PER_XCD;
    if (at >= rounds * PER_XCD) {
        const int last = at - rounds * PER_XCD;
        if (last >= rest / XCDS + (slot < rest % XCDS ? 1 : 0)) return;
        gid = p.first + rounds * NUM_CUS + slot * (rest / XCDS) + min(slot, rest % XCDS) + last;
    }
    int i = 0;
#pragma unroll
    for (int j = 1; j < MIXED_MAX; ++j)
        if (gid >= grp.first[j]) i = j;
    const MixedEntry& e = grp.e[i];
    const int tile = gid - grp.first[i];
#define CHIMERA_MIXED(...)                                                                                                  \
    gemm_ring_tile<__VA_ARGS__, false, false, EPI_ACCUM_F32>(lds, e.a, e.b, nullptr, nullptr, e.c, nullptr, e.m, e.n, grp.k, \
        e.lda, e.ldb, EPI_ACCUM_F32, grp.flags, 0, e.tiles_m, e.tiles_n, e.group_m, tile, e.bsum, false, e.col0, Ahead{nullptr, 0}, e.band)
    if (e.form == TILE_256) CHIMERA_MIXED(256, 256, 2, 4, 1);
    else if (e.form == TILE_128x256) CHIMERA_MIXED(128, 256, 1, 4, 2);
    else if (e.form == TILE_256x128) CHIMERA_MIXED(256, 128, 2, 2, 2);
    else CHIMERA_MIXED(128, 128, 2, 2, 2);
#undef CHIMERA_MIXED
}

// A launch of 256x256 tiles runs in rounds of NUM_CUS tiles, and a last round with few tiles
// costs as much as a full one.  The products here can be cut along m without touching the data
// (row bands of A and C are just pointer offsets), so the last `b` bands of 256 rows may go to a
// second launch with 128x128 tiles instead.  Cost estimate in units of one 256x256 round: a round
// of 128x128 tiles (a quarter of the flops) counts 0.45.  Measured, launch included: 0.36 to 0.39 of a 256x256
// round at one tile per CU (k = 1600: 18.4 against 49.5 us A B, 24.5 against 68 A^T B), 0.34 each of two rounds
// at two per CU; the rest stands for what an estimate in whole rounds leaves out.  Returns the b
// that minimises it (0: leave the product whole).  Columns are counted by the same rule with rows and columns exchanged.
int bands_to_peel(int tm, int tn, int n, double* cost) {
    const int tn128 = (n + 127) / 128;
    auto rounds = [](long tiles) { return (double)((tiles + NUM_CUS - 1) / NUM_CUS); };
    const double whole = rounds((long)tm * tn);
    int best_b = 0;
    double best = whole - 0.25;                                  // a split must pay for its second launch
    for (int b = 1; b < tm; ++b) {
        const double est = rounds((long)(tm - b) * tn) + 0.45 * rounds((long)b * 2 * tn128);
        if (est < best) { best = est; best_b = b; }
    }
    *cost = best;
    return best_b;
}

struct TileChoice { int bm, bn, splits; };

// The kernels' `epi_flag` argument modifies the epilogue: for the GeLU epilogues 1 selects the
// erf form (0: tanh form); for the float-accumulate epilogue it holds ACCUM_* flags, none in a single product
// (ACCUM_OVERWRITE: the column sums replace bsum too).
inline int epilogue_flag(const GemmArgs& g) { return g.epilogue == EPI_ACCUM_F32 ? 0 : g.gelu_erf; }
// A forward that keeps nothing leaves out u, half of what the first product of an MLP writes: six blocks of 1600 at 1264 tokens
// 775 -> 761 us, bert48 with doubled forwards 52.1 -> 51.4 ms.
inline void* result(const GemmArgs& g) { return g.epilogue == EPI_BIAS_GELU && g.c_unused ? nullptr : g.c; }

inline Ahead ahead_of(const GemmArgs& g) { return {(const char*)g.ahead, (unsigned)g.ahead_bytes}; }

// Tuning aids, read from the environment once (first use) and changeable through
// chimera_gemm_tuning(): a forced tile ("256x256", "128x128" or "256x256x<splits>" in
// CHIMERA_GEMM_TILE) and the form of the LDS-DMA kernels (CHIMERA_GEMM_ASYNC: "0" = the
// register-staged kernels, "4k" = the k-sliced 128x128 form always, "2" = never).
enum AsyncMode { ASYNC_AUTO = 0, ASYNC_OFF = 1, ASYNC_KSLICED = 2, ASYNC_PLAIN = 3 };
struct Tuning { TileChoice forced{0, 0, 0}; int async_mode = ASYNC_AUTO; unsigned long long version = 0; };
Tuning& tuning() {
    static Tuning t = [] {
        Tuning v;
        if (const char* e = std::getenv("CHIMERA_GEMM_TILE")) std::sscanf(e, "%dx%dx%d", &v.forced.bm, &v.forced.bn, &v.forced.splits);
        if (const char* e = std::getenv("CHIMERA_GEMM_ASYNC"))
            v.async_mode = e[0] == '0' ? ASYNC_OFF : (!std::strcmp(e, "4k") ? ASYNC_KSLICED : ASYNC_PLAIN);
        return v;
    }();
    return t;
}
TileChoice forced_tile() { return tuning().forced; }

constexpr int MAX_SPLITS = 8;

// gemm_ring_tile addresses a lane's pieces by 32-bit byte offsets from the tile's corner: up to 255 rows away
// in a k-contiguous operand, up to 31 rows of k (as many as there are) and 255 elements in an index-contiguous one.
// Operands that reach further go to the register-staged kernel, whose element offsets reach 2^32.  (A group's never do
// where k is 64 or more: k * ld < 2^32 bounds ld; a stage's rows are at most 16384 elements long.)
bool far_operand(const GemmArgs& g) {
    const long k_rows = std::min(g.k, 32) - 1;
    auto far = [&](int k_contiguous, long ld) { return k_contiguous ? ld >= 1l << 23 : k_rows * ld + 256 >= 1l << 31; };
    return far(g.a_kc, g.lda) || far(g.b_kc, g.ldb);
}

// 64x64 tiles while they all fit on the chip at once, two per CU: a smaller product is bound by
// its chain of latencies and by how many CUs pull its operands, not by the bytes a small tile
// costs.  Measured, 128x128 -> 64x64: 632 x 1600 x 1600 (65 tiles of 128x128, 250 of 64x64) 13.7 -> 9.2 us,
// 632 x 1600 x 6400 55 -> 31, 1024 x 1280 x 5120 (80, 320) 48.6 -> 42.4, 1264 x 1600 x 6400 (130, 500) 55.0 -> 52.3,
// 1024 x 2048 x 2048 (128, 512) 16.2 -> 16.5; beyond it turns: 1024 x 2560 x 640 (160, 640) 9.8 -> 11.9,
// 632 x 4800 x 1600 (190, 750) 17.7 -> 23.9, 1264 x 2400 x 6400 (190, 760) 60.6 -> 82.9.
bool small_tiles(long tiles64) { return tiles64 <= 2 * NUM_CUS && tuning().async_mode == ASYNC_AUTO; }

// The tile of such a product: the largest with which it still has a tile for every CU or nearly so.  A CU takes 60 to 90 bytes a
// nanosecond, so what bounds a small output's k loop is what its few workgroups have to read, (bm + bn) a step each; once
// the chip is full a larger tile reads less in all.  Measured, 64x64 -> 32x32: 256 x 256 x 256 3.74 -> 3.30 us, x 1024 5.5 -> 3.9,
// 400 x 320 x 1280 6.2 -> 4.2, 128 x 1600 x 6400 (200 tiles) 20.1 -> 11.8, 512 x 512 x 2048 (256) 8.2 -> 5.0; 32x64: 1024 x 512 x 2048
// (256) 8.8 -> 7.1 (32x32 8.4), 333 x 776 x 3104 13.7 -> 10.9 (12.4), 400 x 960 x 320 3.9 -> 3.7 (4.0).
// 64x64, two per CU -> 128x64: 1264 x 1600 x 6400 (250) 46.7 -> 39.5, x 1600 13.9 -> 12.1, 1024 x 2048 x 2048 (256) 16.6 -> 14.2,
// 2048 x 768 x 3072 21.5 -> 17.2, 512 x 3072 x 1024 10.7 -> 9.3; beside another stage 10.6 -> 11.1 each at k = 1600, 13.3 -> 12.6 at 2048.
// From k = 128 on: at 64 and 96 it is 1 to 5 % slower (1152 x 1280 x 64 A B 4.21 -> 4.44 us, A B^T 4.27 -> 4.40), at 128 as fast, from 256 on 3 to
// 13 % faster.  With the GeLU derivative, whose epilogue is the longest, from 640 on: x 192 2 to 3 % slower, x 512 1 to 2, x 640 as fast, x 768
// 2 to 4 % faster.
// Beside another stage the tiles below 64x64 may take half of the CUs: they read more in all, and what one stage's tiles take the
// other's do without.  Replays of two stages with the limit at all CUs -> at half: two blocks of 512 at 1024 tokens 1409 -> 1371 us
// (64x64 tiles throughout: 1398), of 512 at 512 1259 -> 1238, of 1024 at 128 1483 -> 1443 and at 256 1728 -> 1684, of 1600 at 128 2610 -> 2538; of 256 at
// 256, whose products need 64 to 192 such tiles, 859 -> 857 (at three quarters of the CUs 853).
// (Weight gradients stay on 64x64 tiles, so that one alone has the bits of one in a group.)
TileChoice small_tile(const GemmArgs& g) {
    if (!g.a_kc) return {64, 64, 1};
    auto fits = [&](int bm, int bn, int cus) { return (long)((g.m + bm - 1) / bm) * ((g.n + bn - 1) / bn) <= cus; };
    const int few = g.beside ? NUM_CUS / 2 : NUM_CUS;
    if (fits(32, 32, few)) return {32, 32, 1};
    if (fits(32, 64, few)) return {32, 64, 1};
    const int long_k = g.beside ? 2048 : g.epilogue == EPI_DGELU ? 640 : 128;
    if (!fits(64, 64, NUM_CUS) && fits(128, 64, NUM_CUS) && g.k >= long_k) return {128, 64, 1};
    return {64, 64, 1};
}

// 256x128 tiles for a product that shares the chip with another stage's: it should then take little of the
// chip's time, not little time.  Alone it is slower than 128x128, whose tiles are twice as many (4096 x 1024 x
// 4096 40 -> 56 us, 2048 x 1600 x 6400 57 -> 82), but it spends a third fewer CU-microseconds, a quarter less
// traffic into LDS and a third less out of it, and the other stage has work for the CUs it leaves.  Replays of
// two stages, 128x128 -> 256x128: bert48 21.1 -> 20.6 ms, gpt2-1p3b-n32 103.4 -> 100.2, gpt2-deep 52.3 -> 50.5, three
// blocks of 2048 at 3000 tokens 13.2 -> 12.7.  With fewer than 100 tiles the two stages together leave the chip
// half empty (1024 wide at 3000 tokens, 96 tiles: 8.2 -> 8.4 ms; 768 at 4096, 96: 7.3 -> 7.5), with k below 1024 the larger
// epilogue weighs more than the loop saves (512 wide at 4096 tokens, 192 tiles: 4.69 -> 4.77).  The two-per-CU form of
// 64x64 tiles (257 to 512 of them) gives way earlier, from 60 tiles on, where k is long: four blocks of 2048 at 1024
// tokens 8.06 -> 7.53 ms, six of 1024 at 2048 tokens 6.71 -> 6.59; not at 512 wide, k up to 2048 (4.69 -> 4.74).
bool wide_tiles(const GemmArgs& g) {
    if (!g.beside || tuning().async_mode != ASYNC_AUTO) return false;
    const long t2 = (long)((g.m + 255) / 256) * ((g.n + 127) / 128), t64 = (long)((g.m + 63) / 64) * ((g.n + 63) / 64);
    if (t2 > NUM_CUS) return false;
    return (t2 >= 100 && g.k >= 1024) || (t2 >= 60 && t64 > NUM_CUS && small_tiles(t64) && g.k > 2048);
}

// 256x256 (8 wavefronts) once the output has enough such tiles for most of the 256 CUs,
// else 128x128 (4 wavefronts, two workgroups per CU); thresholds measured on MI355X.
// A CU fills LDS from L2 at roughly 64 bytes per clock, so a 128x128x64 step (32 KiB for
// 512 clocks of MFMA work) is fed at half the rate the matrix cores could use; 256x256
// halves the bytes per flop, which is why it wins whenever it can occupy the chip.
// Split-K (several workgroups per 256x256 tile, see the kernel) is available on request
// (CHIMERA_GEMM_TILE=256x256x<splits> plus a workspace) but not chosen by default: on
// MI355X the device-wide fences its hand-over needs cost more than the idle CUs.
TileChoice choose_tile(const GemmArgs& g) {
    TileChoice f = forced_tile();
    const long t256 = (long)((g.m + 255) / 256) * ((g.n + 255) / 256);
    if (f.bm) {
        if (f.splits < 1 || f.bm != 256) f.splits = 1;
        f.splits = std::min(f.splits, std::min(MAX_SPLITS, std::max(1, (g.k + BK - 1) / BK)));
        if (f.splits > 1 && (!g.ws || g.ws_bytes < gemm_mfma_workspace_bytes(g.m, g.n, f.splits))) f.splits = 1;
        return f;
    }
    // (measured at 2048 x 4800 x 1600: 152 tiles of 256x256 on 256 CUs take 42 us, 608 of 128x128 48 us)
    if (t256 >= 144) return {256, 256, 1};
    if (wide_tiles(g)) return {256, 128, 1};
    if (small_tiles((long)((g.m + 63) / 64) * ((g.n + 63) / 64))) return small_tile(g);
    return {128, 128, 1};
}

template <int BM, int BN, int WGM, int WGN, int PF>
int launch_layout(const GemmArgs& g, int splits, hipStream_t s) {
    const int tm = (g.m + BM - 1) / BM, tn = (g.n + BN - 1) / BN;
    const dim3 grid(tm * tn * splits), block(WGM * WGN * 64);
    unsigned* arrivals = (unsigned*)g.ws;                               // [tiles], zero between launches
    float* slabs = g.ws ? (float*)((char*)g.ws + SPLITK_COUNTER_BYTES) : nullptr;
#define CHIMERA_GEMM_LAUNCH(AKC, BKC)                                                                              \
    hipLaunchKernelGGL((gemm_bf16_kernel<BM, BN, WGM, WGN, PF, AKC, BKC>), grid, block, 0, s, (const bf16_t*)g.a,  \
                       (const bf16_t*)g.b, (const bf16_t*)g.bias, (const bf16_t*)g.r, result(g), (bf16_t*)g.c2, g.m, g.n, \
                       g.k, g.lda, g.ldb, g.epilogue, epilogue_flag(g), (g.r_f32 ? 1 : 0) | (g.c_f32 ? 2 : 0), tm, tn,    \
                       splits, slabs, arrivals)
    if (g.a_kc && !g.b_kc) CHIMERA_GEMM_LAUNCH(true, false);
    else if (g.a_kc && g.b_kc) CHIMERA_GEMM_LAUNCH(true, true);
    else CHIMERA_GEMM_LAUNCH(false, false);
#undef CHIMERA_GEMM_LAUNCH
    CHIMERA_LAUNCH_CHECK("bf16 gemm");
    return CHIMERA_OK;
}

template <int BM, int BN, int WGM, int WGN, int WGK, int NS, int SPS = 1>
int launch_async(const GemmArgs& g, hipStream_t s) {
    const int tm = (g.m + BM - 1) / BM, tn = (g.n + BN - 1) / BN;
    const dim3 grid(tm * tn), block(WGM * WGN * WGK * 64);
    const int gm = raster_group(tm, tn, (tm * tn + 7) / 8, BM, BN);
#define CHIMERA_GEMM_LAUNCH(AKC, BKC)                                                                                \
    hipLaunchKernelGGL((gemm_bf16_async_kernel<BM, BN, WGM, WGN, WGK, NS, SPS, AKC, BKC>), grid, block, 0, s,                   \
                       (const bf16_t*)g.a, (const bf16_t*)g.b, (const bf16_t*)g.bias, (const bf16_t*)g.r, result(g), \
                       (bf16_t*)g.c2, g.m, g.n, g.k, g.lda, g.ldb, g.epilogue, epilogue_flag(g),                            \
                       (g.r_f32 ? 1 : 0) | (g.c_f32 ? 2 : 0), tm, tn, gm, ahead_of(g))
    if (g.a_kc && !g.b_kc) CHIMERA_GEMM_LAUNCH(true, false);
    else if (g.a_kc && g.b_kc) CHIMERA_GEMM_LAUNCH(true, true);
    else if constexpr (BM == 64 && BN == 64) CHIMERA_GEMM_LAUNCH(false, false);
    else return fail(CHIMERA_EINVAL, "no %dx%d tile for weight gradients", BM, BN);
#undef CHIMERA_GEMM_LAUNCH
    CHIMERA_LAUNCH_CHECK("bf16 gemm (async)");
    return CHIMERA_OK;
}

// Columns [col0, col0 + 256 * cols256) of the product, or from col0 on.
template <int BM, int BN, int WGM, int WGN, int WGK>
int launch_ring(const GemmArgs& g, hipStream_t s, int col0 = 0, int cols256 = 0) {
    const int tm = (g.m + BM - 1) / BM, tn = cols256 ? cols256 * (256 / BN) : (g.n - col0 + BN - 1) / BN;
    const dim3 grid(tm * tn), block(WGM * WGN * WGK * 64);
    constexpr int PER_CU = RingLds<BM, BN, WGM, WGN, WGK>::PER_CU;
    const int band = raster_band(tm, tn, NUM_CUS * PER_CU, (size_t)g.n * g.k * sizeof(bf16_t));
    const int gm = raster_group(tm, band ? band : tn, std::min((tm * tn + 7) / 8, PER_XCD * PER_CU), BM, BN);
#define CHIMERA_GEMM_LAUNCH(AKC, BKC)                                                                                \
    hipLaunchKernelGGL((gemm_bf16_ring_kernel<BM, BN, WGM, WGN, WGK, AKC, BKC>), grid, block, 0, s,                     \
                       (const bf16_t*)g.a, (const bf16_t*)g.b, (const bf16_t*)g.bias, (const bf16_t*)g.r, result(g), \
                       (bf16_t*)g.c2, g.m, g.n, g.k, g.lda, g.ldb, g.epilogue, epilogue_flag(g),                            \
                       (g.r_f32 ? 1 : 0) | (g.c_f32 ? 2 : 0), tm, tn, gm, band, col0, ahead_of(g))
    if (g.a_kc && !g.b_kc) CHIMERA_GEMM_LAUNCH(true, false);
    else if (g.a_kc && g.b_kc) CHIMERA_GEMM_LAUNCH(true, true);
    else CHIMERA_GEMM_LAUNCH(false, false);
#undef CHIMERA_GEMM_LAUNCH
    CHIMERA_LAUNCH_CHECK("bf16 gemm (ring)");
    return CHIMERA_OK;
}

// Name of the kernel instantiation the last grouped launch on this thread went to (for reports).
thread_local char g_last_group_kernel[96] = "";
void note_group_kernel(const char* name) { std::snprintf(g_last_group_kernel, sizeof g_last_group_kernel, "%s", name); }

template <int BM, int BN, int WGM, int WGN, int WGK>
int launch_group_ring(const GemmGroup& grp, hipStream_t s) {
    char name[96];
    std::snprintf(name, sizeof name, "gemm_bf16_ring_group_kernel<%d,%d,%d,%d,%d>", BM, BN, WGM, WGN, WGK);
    note_group_kernel(name);
    hipLaunchKernelGGL((gemm_bf16_ring_group_kernel<BM, BN, WGM, WGN, WGK>), dim3(grp.first[grp.count]), dim3(WGM * WGN * WGK * 64), 0, s, grp);
    CHIMERA_LAUNCH_CHECK("bf16 gemm group");
    return CHIMERA_OK;
}

template <int BM, int BN, int WGM, int WGN, int WGK, int NS, int SPS = 1>
int launch_group(const GemmGroup& grp, hipStream_t s) {
    char name[96];
    std::snprintf(name, sizeof name, "gemm_bf16_async_group_kernel<%d,%d,%d,%d,%d,%d,%d,false,false>", BM, BN, WGM, WGN, WGK, NS, SPS);
    note_group_kernel(name);
    const dim3 grid(grp.first[grp.count]), block(WGM * WGN * WGK * 64);
    hipLaunchKernelGGL((gemm_bf16_async_group_kernel<BM, BN, WGM, WGN, WGK, NS, SPS, false, false>), grid, block, 0, s, grp);
    CHIMERA_LAUNCH_CHECK("bf16 gemm group");
    return CHIMERA_OK;
}

// A group on tiles of 256x256, its remainders of up to 128 rows or columns on halves of them, begun first, and what full rounds leave
// over on quarters or halves, begun last.  Against 256x256 tiles throughout, with the last row bands of one product in a launch of
// 128x128 tiles of its own: blocks of 1280, 1344, 1408, 1600 and 1792 at 2048 tokens 106 -> 103, 132 -> 109, 137 -> 116, 169 -> 152 and 207 -> 188 us;
// of 1024, 1536 and 2048, which have neither remainders nor a rest, within 1 %.  gpt2-1p3b-n32 96.0 -> 93.6 ms.
// (1) A remainder costs a half tile, not a whole one: a block of 1600 needs 450 + 82 halves instead of 532.
// (2) All workgroups of a launch that starts with one size reach their epilogues together, and the chip then waits for HBM: 256 tiles of += x 64
// take 25.5 us, 16 take 10.7.  Halves first put CUs out of step, and give CUs to the other lane of a replay at other times than the
// rest: halves first -> last gpt2-1p3b-n32 94.2 -> 96.1 ms, six blocks of 1600 at 632 tokens, forward and backward, 1665 -> 1706 us.  Halving
// whole tiles for it does not pay: a half takes 0.6 of a tile's time (2048 wide, 128 of 768 halved 222 -> 235 us).
// (3) Up to 64 tiles beyond full rounds take a round of quarters, 0.38 of one of 256x256; more of them a round of halves where these and
// the remainders' fit into one.
int launch_group_mixed(int count, const GemmArgs* g, float* const* bsum, int overwrite, bool smaller, hipStream_t stream) {
    int fm[GROUP_MAX], fn[GROUP_MAX], cut_m[GROUP_MAX] = {}, cut_n[GROUP_MAX] = {};      // tile rows and columns of 256x256, how many of each are cut smaller
    long full = 0, half = 0;
    for (int i = 0; i < count; ++i) {
        const int rm = g[i].m % 256, rn = g[i].n % 256;
        fm[i] = g[i].m / 256 + (rm > (smaller ? 128 : 0));
        fn[i] = g[i].n / 256 + (rn > (smaller ? 128 : 0));
        full += (long)fm[i] * fn[i];
        if (fm[i] * 256 < g[i].m) half += (g[i].n + 255) / 256;
        if (fn[i] * 256 < g[i].n) half += fm[i];
    }
    const long over = smaller && full + half > NUM_CUS ? (full + half) % NUM_CUS : 0;
    const bool quarters = 4 * over <= NUM_CUS;
    const long left = full % NUM_CUS;                        // of the whole tiles alone
    const bool fill = smaller && !quarters && full > NUM_CUS && half + 2 * left <= NUM_CUS;
    const long todo = fill ? left : over <= full && (quarters || (over > half && 2 * over <= NUM_CUS)) ? over : 0;
    const long most = quarters ? NUM_CUS / 4 : (NUM_CUS - (fill ? half : 0)) / 2;
    // Whole bands of rows or columns of one product, or bands of two kinds where that does not do, that come to `todo` tiles or the fewest
    // more, and to a round of the smaller tiles at most; less than `todo` would leave the last round as it is.  With one kind only, which
    // may find nothing, -> so: a block of 2696 at 2048 tokens (117 tiles) 435 -> 420 us, 1496 x 13464 x 2048 (62: a row of 53, two columns
    // of 5) 111 -> 91; but with two kinds wherever they come nearer a block of 1152 (19 tiles in place of 20) 78 -> 88.
    auto tiles_of = [&](int i, bool rows) { return (long)(rows ? fn[i] - cut_n[i] : fm[i] - cut_m[i]); };
    auto bands_of = [&](int i, bool rows) { return (long)(rows ? fm[i] - cut_m[i] : fn[i] - cut_n[i]); };
    auto take = [&](int i, bool rows, long bands) { (rows ? cut_m : cut_n)[i] += (int)bands; };
    struct Bands { int i; bool rows; long count; } first{}, last{}, none{};
    long best = most + 1;
    auto finish = [&](const Bands& before, long got) {
        for (int i = 0; i < count; ++i)
            for (bool rows : {true, false}) {
                const long per = tiles_of(i, rows), bands = per > 0 ? (todo - got + per - 1) / per : 0;
                if (bands > 0 && bands <= bands_of(i, rows) && got + bands * per < best) { best = got + bands * per; first = before; last = {i, rows, bands}; }
            }
    };
    if (todo > 0) {
        finish(none, 0);
        if (best > most)
            for (int i = 0; i < count; ++i)
                for (bool rows : {true, false}) {
                    const long per = tiles_of(i, rows), bands = per > 0 ? std::min(todo / per, bands_of(i, rows)) : 0;
                    if (bands <= 0) continue;
                    take(i, rows, bands);
                    finish({i, rows, bands}, bands * per);
                    take(i, rows, -bands);
                }
        take(first.i, first.rows, first.count);
        take(last.i, last.rows, last.count);
    }
    MixedGroup grp{};
    grp.k = g[0].k; grp.flags = (overwrite ? ACCUM_OVERWRITE : 0) | (g[0].c_once ? ACCUM_ONCE : 0);
    std::fill(std::begin(grp.first), std::end(grp.first), INT_MAX);
    int tiles = 0;
    auto put = [&](int i, int form, int row0, int rows, int col0, int cols) {
        if (rows <= 0 || cols <= 0) return;
        const int bm = form == TILE_128x256 || form == TILE_128 ? 128 : 256, bn = form == TILE_256x128 || form == TILE_128 ? 128 : 256;
        MixedEntry& e = grp.e[grp.count++];
        e.a = (const bf16_t*)g[i].a + row0;                      // A is [k, m]
        e.b = (const bf16_t*)g[i].b;
        e.c = (float*)g[i].c + (size_t)row0 * g[i].n;
        e.bsum = bsum && row0 == 0 ? bsum[i] : nullptr;
        e.m = rows; e.n = g[i].n; e.lda = g[i].lda; e.ldb = g[i].ldb; e.col0 = col0;
        e.tiles_m = (rows + bm - 1) / bm; e.tiles_n = (cols + bn - 1) / bn;
        e.form = form; grp.first[&e - grp.e] = tiles;
        tiles += e.tiles_m * e.tiles_n;
    };
    int local = 0;
    auto close = [&](int h) {                                    // the entries put since the last call are phase h
        MixedPhase& p = grp.phase[h];
        p.first = h ? grp.phase[h - 1].first + grp.phase[h - 1].tiles : 0;
        p.tiles = tiles - p.first; p.local = local; p.skew = p.first % XCDS;
        local += (p.tiles + XCDS - 1) / XCDS;
        for (int i = 0; i < grp.count; ++i) {
            MixedEntry& e = grp.e[i];
            if (grp.first[i] < p.first) continue;
            const int bm = e.form == TILE_128x256 || e.form == TILE_128 ? 128 : 256, bn = e.form == TILE_256x128 || e.form == TILE_128 ? 128 : 256;
            e.band = raster_band(e.tiles_m, e.tiles_n, NUM_CUS, (size_t)e.n * grp.k * sizeof(bf16_t));
            e.group_m = raster_group(e.tiles_m, e.band ? e.band : e.tiles_n, std::min((p.tiles + XCDS - 1) / XCDS, PER_XCD), bm, bn);
        }
    };
    // rows [0, whole_m) of columns [0, whole_n) on 256x256 tiles, up to `rows` and `cols` cut smaller, then the remainders
    auto rows = [&](int i) { return std::min(fm[i] * 256, g[i].m); };
    auto cols = [&](int i) { return std::min(fn[i] * 256, g[i].n); };
    auto whole_m = [&](int i) { return std::min((fm[i] - cut_m[i]) * 256, g[i].m); };
    auto whole_n = [&](int i) { return std::min((fn[i] - cut_n[i]) * 256, g[i].n); };
    for (int i = 0; i < count; ++i) put(i, TILE_128x256, rows(i), g[i].m - rows(i), 0, g[i].n);
    for (int i = 0; i < count; ++i) put(i, TILE_256x128, 0, rows(i), cols(i), g[i].n - cols(i));
    close(0);
    for (int i = 0; i < count; ++i) put(i, TILE_256, 0, whole_m(i), 0, whole_n(i));
    close(1);
    for (int i = 0; i < count; ++i) {
        put(i, quarters ? TILE_128 : TILE_128x256, whole_m(i), rows(i) - whole_m(i), 0, whole_n(i));
        put(i, quarters ? TILE_128 : TILE_256x128, 0, rows(i), whole_n(i), cols(i) - whole_n(i));
    }
    close(2);
    hipLaunchKernelGGL(gemm_bf16_mixed_group_kernel, dim3(local * XCDS), dim3(512), 0, stream, grp);
    CHIMERA_LAUNCH_CHECK("bf16 gemm group");
    return CHIMERA_OK;
}

}  // namespace

bool gemm_mfma_supports(const GemmArgs& g) {
    if (!g.a_kc && g.b_kc) return false;                       // layout no linear layer needs
    if ((g.n % 8) || (g.lda % 8) || (g.ldb % 8)) return false;
    if ((g.a_kc || g.b_kc) && (g.k % 8)) return false;         // index-contiguous operands are masked row by row: any k
    if (!g.a_kc && (g.m % 8)) return false;
    if (((uintptr_t)g.a | (uintptr_t)g.b) & 15) return false;  // 16-byte vector loads
    // operand elements are addressed with 32-bit offsets
    const unsigned long long ea = (unsigned long long)(g.a_kc ? g.m : g.k) * g.lda, eb = (unsigned long long)(g.b_kc ? g.n : g.k) * g.ldb;
    if (ea >= (1ull << 32) || eb >= (1ull << 32)) return false;
    return g.m >= 1 && g.n >= 1 && g.k >= 1;
}

// Workspace of a split-K launch: arrival counters (zero before the first launch, left zero
// by every launch) followed by one float slab per (split, 256x256 tile).
size_t gemm_mfma_workspace_bytes(int m, int n, int splits) {
    const size_t tiles = (size_t)((m + 255) / 256) * ((n + 255) / 256);
    return SPLITK_COUNTER_BYTES + (size_t)splits * tiles * 256 * 256 * sizeof(float);
}
// Workspace that allows any split count up to MAX_SPLITS for an m x n output.
size_t gemm_mfma_workspace_need(int m, int n, int k) {
    if (m < 1 || n < 1 || k < 1) return 0;
    return gemm_mfma_workspace_bytes(m, n, MAX_SPLITS);
}

int gemm_mfma_bf16(const GemmArgs& g, void* stream) {
    if (!gemm_mfma_supports(g)) return fail(CHIMERA_EINVAL, "bf16 matrix-core gemm: unsupported shape or layout");
    if (g.epilogue < EPI_NONE || g.epilogue > EPI_ACCUM_F32) return fail(CHIMERA_EINVAL, "unknown epilogue %d", g.epilogue);
    hipStream_t s = (hipStream_t)stream;
    const bool far = far_operand(g);
    TileChoice t = choose_tile(g);
    if (far && (t.bm < 128 || t.bm != t.bn)) t = {128, 128, 1};
    if (t.splits > 1 && (size_t)((g.m + 255) / 256) * ((g.n + 255) / 256) * sizeof(unsigned) > SPLITK_COUNTER_BYTES)
        return fail(CHIMERA_EINVAL, "too many tiles for split-K");
    // 128x128 tiles: with one workgroup per CU, a workgroup of 4 wavefronts leaves one wavefront
    // per SIMD, and nothing covers its LDS latency and the barrier of every k step; then 8
    // wavefronts share the tile, two per 64x64 block (their partial sums meet in LDS at the end),
    // over a ring of 128 KiB - one such workgroup per CU, so more than NUM_CUS tiles would take it
    // two rounds.  Beyond that the 4-wavefront form with its two buffers (64 KiB of LDS, two
    // workgroups per CU) is faster.
    const int mode = tuning().async_mode;
    const bool can_async = t.splits == 1 && mode != ASYNC_OFF && !far;
    if (can_async) {
        if (t.bm == 256 && t.bn == 256) {
            if (!g.a_kc && g.epilogue == EPI_ACCUM_F32) return launch_group_mixed(1, &g, nullptr, 0, forced_tile().bm == 0, s);
            const int tm = (g.m + 255) / 256, tn = (g.n + 255) / 256;
            double by_rows = 0, by_columns = 0;
            const int b = forced_tile().bm ? 0 : bands_to_peel(tm, tn, g.n, &by_rows);
            const int bc = forced_tile().bm ? 0 : bands_to_peel(tn, tm, g.m, &by_columns);
            if (bc > 0 && by_columns < by_rows && g.n - (tn - bc) * 256 >= 8) {
                // columns in the same way: wide outputs of few tile rows (1024 x 50304 x 4096, 788 tiles:
                // three full rounds and 20 tiles: 386 -> 344 us)
                const int col0 = (tn - bc) * 256;
                GemmArgs head = g;
                head.ahead = nullptr; head.ahead_bytes = 0;
                if (int rc = launch_ring<256, 256, 2, 4, 1>(head, s, 0, tn - bc)) return rc;
                if ((long)((g.m + 127) / 128) * ((g.n - col0 + 127) / 128) <= NUM_CUS) return launch_ring<128, 128, 2, 2, 2>(g, s, col0);
                return launch_ring<128, 128, 2, 2, 1>(g, s, col0);
            }
            if (b > 0 && g.m - (tm - b) * 256 >= 8) {
                // rows [0, m0) with 256x256 tiles, rows [m0, m) with 128x128 tiles
                const size_t m0 = (size_t)(tm - b) * 256;
                const size_t csz = (g.epilogue == EPI_ACCUM_F32 || g.c_f32) ? 4 : 2;
                GemmArgs head = g, tail = g;
                head.ahead = nullptr; head.ahead_bytes = 0;
                head.m = (int)m0;
                tail.m = g.m - (int)m0;
                tail.a = (const char*)g.a + (g.a_kc ? m0 * g.lda : m0) * 2;
                tail.c = (char*)g.c + m0 * g.n * csz;
                if (g.c2) tail.c2 = (char*)g.c2 + m0 * g.n * 2;
                if (g.r) tail.r = (const char*)g.r + m0 * g.n * (g.r_f32 ? 4 : 2);
                if (int rc = launch_ring<256, 256, 2, 4, 1>(head, s)) return rc;
                const long t128 = (long)((tail.m + 127) / 128) * ((tail.n + 127) / 128);
                if (t128 <= NUM_CUS) return launch_ring<128, 128, 2, 2, 2>(tail, s);
                return launch_ring<128, 128, 2, 2, 1>(tail, s);
            }
            return launch_ring<256, 256, 2, 4, 1>(g, s);
        }
        if (t.bm == 256) return launch_ring<256, 128, 2, 2, 2>(g, s);
        if (t.bm == 128 && t.bn == 64) return launch_async<128, 64, 2, 2, 2, 6, 2>(g, s);
        if (t.bm == 32) return t.bn == 32 ? launch_async<32, 32, 1, 1, 4, 8, 2>(g, s) : launch_async<32, 64, 1, 2, 2, 8, 2>(g, s);
        if (t.bm == 64) {
            // one tile per CU at most: all of LDS for one workgroup, an eight-stage ring walked two stages per
            // barrier by two wavefronts per SIMD (256 x 256 x 1024: 6.7 -> 6.1 us; 632 x 1600 x 6400: 28.4 -> 25.4)
            if ((long)((g.m + 63) / 64) * ((g.n + 63) / 64) <= NUM_CUS) return launch_async<64, 64, 2, 2, 2, 8, 2>(g, s);
            return launch_async<64, 64, 1, 2, 2, 4>(g, s);
        }
        if (t.bm == 128 && t.bn == 128) {
            const long t128 = (long)((g.m + 127) / 128) * ((g.n + 127) / 128);
            const bool ksplit = mode != ASYNC_AUTO ? mode == ASYNC_KSLICED : t128 <= NUM_CUS;
            if (ksplit) return launch_ring<128, 128, 2, 2, 2>(g, s);
            return launch_ring<128, 128, 2, 2, 1>(g, s);
        }
    }
    if (t.bm == 256 && t.bn == 256) return launch_layout<256, 256, 2, 4, 1>(g, t.splits, s);
    if (t.bm == 128 && t.bn == 128) return launch_layout<128, 128, 2, 2, 1>(g, 1, s);
    return fail(CHIMERA_EINVAL, "no %dx%d gemm tile", t.bm, t.bn);
}

// How a product of k-contiguous operands is cut along k (splits = 1: not at all): fewer tiles than CUs leave
// CUs idle, and 256x256 tiles cost a third less energy and time per flop than the 128x128 tiles that an uncut
// product of 64 to 143 of them takes.  Model of the time in us, constants measured: a step of 64 k of a round of
// tiles (A B^T, k 1024 to 8192: 256x256 1.55 to 1.63 from random operands that miss the caches, 128x128 0.50 to 0.56, 64x64
// 0.18 to 0.30), against the float slabs written and read (at 4.5 TB/s) and the launch that adds them.
// 4096 x 1024 x 50304 462 -> 355 + 12 us; a head's whole pass over 1000 x 512 x 20000 164 -> 131, 128 x 128 x 65536
// 252 -> 87, 1111 x 776 x 50304 507 -> 443, 632 x 1600 x 50304 589 -> 515 us.
struct SplitPlan { int tile, splits, k_per; };
static SplitPlan split_plan(int m, int n, int k) {
    const long steps = (k + RK - 1) / RK, t256 = (long)((m + 255) / 256) * ((n + 255) / 256), t128 = (long)((m + 127) / 128) * ((n + 127) / 128);
    const long t64 = (long)((m + 63) / 64) * ((n + 63) / 64);
    SplitPlan best{0, 1, k};
    if (forced_tile().bm || tuning().async_mode != ASYNC_AUTO || t256 >= 144) return best;
    constexpr double STEP256 = 1.4, STEP128 = 0.5, STEP64 = 0.25, SLAB = 8 / 4.5e6, LAUNCH = 10;
    auto rounds = [](long tiles) { return (double)((tiles + NUM_CUS - 1) / NUM_CUS); };
    double cost = steps * (t64 <= 2 * NUM_CUS ? rounds(t64) * STEP64 : rounds(t128) * STEP128);
    cost *= 0.9;                                         // a split must pay clearly
    for (int s = 2; s <= 64 && steps / s >= 8; ++s) {
        const long per = (steps + s - 1) / s;
        if ((steps + per - 1) / per != s) continue;
        const double slabs = SLAB * s * m * n + LAUNCH;
        const double c256 = rounds(t256 * s) * per * STEP256 + slabs, c128 = rounds(t128 * s) * per * STEP128 + slabs;
        if (c256 < cost) { cost = c256; best = {256, s, (int)per * RK}; }
        if (c128 < cost) { cost = c128; best = {128, s, (int)per * RK}; }
    }
    return best;
}
size_t gemm_mfma_split_bytes(int m, int n, int k) {
    const SplitPlan p = split_plan(m, n, k);
    return p.splits > 1 ? (size_t)p.splits * m * n * sizeof(float) : 0;
}
int gemm_mfma_split(const GemmArgs& g, float* slabs, void* stream) {
    if (!gemm_mfma_supports(g) || !g.a_kc || !g.b_kc || g.epilogue != EPI_NONE || ((uintptr_t)g.c | (uintptr_t)slabs) & 15)
        return fail(CHIMERA_EINVAL, "split product: k-contiguous operands and a plain bf16 result");
    const SplitPlan p = split_plan(g.m, g.n, g.k);
    if (p.splits < 2 || far_operand(g)) return gemm_mfma_bf16(g, stream);
    hipStream_t s = (hipStream_t)stream;
    const int tm = (g.m + p.tile - 1) / p.tile, tn = (g.n + p.tile - 1) / p.tile;
    const int gm = raster_group(tm, tn, std::min(tm * tn, (tm * tn * p.splits + 7) / 8), p.tile, p.tile);
    const dim3 grid(tm * tn * p.splits), block(512);
#define CHIMERA_SPLIT_LAUNCH(...)                                                                                       \
    hipLaunchKernelGGL((gemm_bf16_ring_split_kernel<__VA_ARGS__>), grid, block, 0, s, (const bf16_t*)g.a, (const bf16_t*)g.b, \
                       slabs, g.m, g.n, g.k, g.lda, g.ldb, tm, tn, gm, p.splits, p.k_per)
    if (p.tile == 256) CHIMERA_SPLIT_LAUNCH(256, 256, 2, 4, 1);
    else CHIMERA_SPLIT_LAUNCH(128, 128, 2, 2, 2);
#undef CHIMERA_SPLIT_LAUNCH
    CHIMERA_LAUNCH_CHECK("bf16 gemm (split)");
    const size_t elems = (size_t)g.m * g.n;
    hipLaunchKernelGGL(split_sum_kernel, dim3((unsigned)((elems / 8 + 255) / 256)), dim3(256), 0, s, slabs, elems, p.splits, (bf16_t*)g.c);
    CHIMERA_LAUNCH_CHECK("split sum");
    return CHIMERA_OK;
}

bool gemm_mfma_group_supports(int count, const GemmArgs* g) {
    if (count < 1 || count > GROUP_MAX || !g) return false;
    for (int i = 0; i < count; ++i) {
        if (g[i].a_kc || g[i].b_kc || g[i].epilogue != EPI_ACCUM_F32 || !gemm_mfma_supports(g[i])) return false;
        if (g[i].k != g[0].k) return false;
        if ((uintptr_t)g[i].c & 15) return false;
    }
    return true;
}

namespace {
int launch_group_tiled(int count, const GemmArgs* g, float* const* bsum, int overwrite, int tile, hipStream_t stream) {
    GemmGroup grp{};
    grp.count = count; grp.k = g[0].k; grp.overwrite = overwrite ? 1 : 0;
    int tiles = 0;
    for (int i = 0; i < count; ++i) {
        grp.a[i] = (const bf16_t*)g[i].a; grp.b[i] = (const bf16_t*)g[i].b; grp.c[i] = (float*)g[i].c;
        grp.bsum[i] = bsum ? bsum[i] : nullptr;
        grp.m[i] = g[i].m; grp.n[i] = g[i].n; grp.lda[i] = g[i].lda; grp.ldb[i] = g[i].ldb;
        grp.tiles_m[i] = (g[i].m + tile - 1) / tile; grp.tiles_n[i] = (g[i].n + tile - 1) / tile;
        grp.first[i] = tiles;
        tiles += grp.tiles_m[i] * grp.tiles_n[i];
    }
    for (int i = 0; i < count; ++i) grp.group_m[i] = raster_group(grp.tiles_m[i], grp.tiles_n[i], (tiles + 7) / 8, tile, tile);
    for (int i = count; i <= GROUP_MAX; ++i) grp.first[i] = tiles;
    if (tile == 64) return tiles <= NUM_CUS ? launch_group<64, 64, 2, 2, 2, 8, 2>(grp, stream) : launch_group<64, 64, 1, 2, 2, 4>(grp, stream);
    // two workgroups per CU or the k-sliced 8-wavefront form
    const int mode = tuning().async_mode;
    const bool ksplit = mode != ASYNC_AUTO ? mode == ASYNC_KSLICED : tiles <= NUM_CUS;
    if (ksplit) return launch_group_ring<128, 128, 2, 2, 2>(grp, stream);
    return launch_group_ring<128, 128, 2, 2, 1>(grp, stream);
}
}  // namespace

int gemm_mfma_bf16_group(int count, const GemmArgs* g, float* const* bsum, int overwrite, void* stream) {
    if (!gemm_mfma_group_supports(count, g))
        return fail(CHIMERA_EINVAL, "bf16 gemm group: 1..%d float-accumulating products with index-contiguous operands, "
                    "one contraction length", GROUP_MAX);
    // tile choice as for single products: 256x256 once such tiles occupy most of the chip, else
    // 128x128.  (192 tiles of 256x256 on 256 CUs beat 768 tiles of 128x128: they pull half the
    // bytes from L2 into LDS, which is what limits these kernels, and the CUs they leave free
    // serve the launches of the other stream.)
    long t256 = 0, t64 = 0;
    for (int i = 0; i < count; ++i) {
        t256 += (long)((g[i].m + 255) / 256) * ((g[i].n + 255) / 256);
        t64 += (long)((g[i].m + 63) / 64) * ((g[i].n + 63) / 64);
    }
    const int forced = forced_tile().bm;
    const int tile = forced == 256 || forced == 128 ? forced : t256 >= 160 ? 256 : small_tiles(t64) ? 64 : 128;
    if (tile == 256) {
        note_group_kernel("gemm_bf16_mixed_group_kernel");
        return launch_group_mixed(count, g, bsum, overwrite, forced == 0, (hipStream_t)stream);
    }
    return launch_group_tiled(count, g, bsum, overwrite, tile, (hipStream_t)stream);
}

const char* gemm_mfma_last_group_kernel() { return g_last_group_kernel; }

int gemm_mfma_set_tuning(int bm, int bn, int splits, int async_mode) {
    if (!((bm == 0 && bn == 0) || (bm == 128 && bn == 128) || (bm == 256 && bn == 256)))
        return fail(CHIMERA_EINVAL, "forced tile %dx%d: 0x0 (automatic), 128x128 or 256x256", bm, bn);
    if (splits < 0 || splits > MAX_SPLITS) return fail(CHIMERA_EINVAL, "splits=%d outside [0,%d]", splits, MAX_SPLITS);
    if (async_mode < ASYNC_AUTO || async_mode > ASYNC_PLAIN) return fail(CHIMERA_EINVAL, "async_mode=%d outside [0,3]", async_mode);
    Tuning& t = tuning();
    t.forced = TileChoice{bm, bn, splits};
    t.async_mode = async_mode;
    ++t.version;
    return CHIMERA_OK;
}

unsigned long long gemm_mfma_tuning_version() { return tuning().version; }

}  // namespace chimera
