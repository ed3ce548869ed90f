// Attention over packed sequences, forward and backward: sequences of different lengths lie behind one another as rows of q, k, v, and every key and
// value head serves a group of neighbouring query heads.  bf16 on the bf16 matrix instructions (head dimensions that are multiples of 8 up to 128,
// compiled for 64 and 128), float on the float ones (multiples of 4).  With S the scores of one sequence and head:
//
//   S = scale q k^T (key <= query under the causal mask),  lse = log sum exp S,  P = exp(S - lse),  ctx = P v
//   delta = rowsum(dctx ctx),  dS = P (dctx v^T - delta),  dq = scale dS k,  dk = scale sum_group dS^T q,  dv = sum_group P^T dctx
//
// The tiles, operand layouts and softmax are those of attention over equal sequences (attention_mfma.hip, attention_f32.hip).  What differs:
//  - A workgroup finds its tile from the offsets in device memory (packed_tile): the grid holds a slot for every tile that `tokens` rows in `seqs`
//    sequences can have, so that a recorded launch serves every packing of the same sizes.
//  - Rows are fetched within the sequence only (beyond its end its last row again), so what other sequences hold, and what lies behind the last, is never read.
//  - dK and dV of a tile sum over the group's heads in the accumulators, in a fixed order.  Where key and value heads are few, the heads
//    of a group are dealt to several workgroups, each with a float slab, which a last kernel adds up.
#include "attention_tiles.h"
#include "spans.h"

#include <type_traits>

namespace chimera {

namespace {

struct PackedArgs {
    const int* offsets;
    int seqs, tokens, heads, kv_heads, group, d;
    float scale;
    const void *q, *k, *v;
    int ldq, ldk, ldv;
    void* ctx;               // out in the forward, in in the backward
    int ldctx;
    float* lse;              // [heads, tokens]
    const void* dctx;
    int lddctx;
    void *dq, *dk, *dv;
    int lddq, lddk, lddv;
    float* delta;            // [heads, tokens]
    float* slabs;            // [splits][2: dk, dv][tokens][kv_heads * d], where splits > 1
    int splits;              // workgroups among which the heads of a group are dealt
};

// ------------------------------------------------------------ which tile is mine
// inclusive prefix sum over the wavefront, all lanes active: within rows of sixteen, then across them
__device__ __forceinline__ int wave_scan(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);     // row_shr:1
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);     // row_bcast:15 into rows 1 and 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);     // row_bcast:31 into rows 2 and 3
    return v;
}
__device__ __forceinline__ int wave_total(int v) { return __builtin_amdgcn_readlane(wave_scan(v), 63); }

// The slot-th tile of ROWS rows of all sequences: first row and length of its sequence and its place there; false where there are fewer tiles.
// SORTED, up to 64 sequences (one a lane): by the tile's place, last places first.  Under the causal mask a tile's work grows with its place (that of a tile of
// keys falls: `at` counts from the sequence's end there), so the longest tiles of all sequences start first.  Otherwise sequence after sequence.
// Offsets are held to [0, tokens] and to be ascending, whatever is in memory.
template <int ROWS, bool SORTED>
__device__ __forceinline__ bool packed_tile(const int* __restrict__ offsets, int seqs, int tokens, int slot, int lane, int& begin, int& len, int& at) {
    int lo = 0, n = 0;
    auto load = [&](int b) {
        lo = 0; n = 0;
        if (b < seqs) {
            lo = min(max(offsets[b], 0), tokens);
            n = min(max(offsets[b + 1], lo), tokens) - lo;
        }
    };
    if (SORTED && seqs <= WAVE) {
        load(lane);
        const int tiles = (n + ROWS - 1) / ROWS;
        auto from = [&](int t) { return wave_total(max(tiles - t, 0)); };       // tiles at places t and later
        if (slot >= from(0)) return false;
        int t = 0;
        for (int step = 1 << (31 - __builtin_clz((tokens + ROWS - 1) / ROWS)); step; step >>= 1)
            if (from(t + step) > slot) t += step;
        slot -= from(t + 1);
        const unsigned long long there = __builtin_amdgcn_ballot_w64(tiles > t);
        const int before = __builtin_amdgcn_mbcnt_hi((unsigned)(there >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)there, 0));
        const int b = __builtin_ctzll(__builtin_amdgcn_ballot_w64(tiles > t && before == slot));
        begin = __builtin_amdgcn_readlane(lo, b);
        len = __builtin_amdgcn_readlane(n, b);
        at = t;
        return true;
    }
    for (int b0 = 0; b0 < seqs; b0 += WAVE) {
        load(b0 + lane);
        const int tiles = (n + ROWS - 1) / ROWS, upto = wave_scan(tiles), all = __builtin_amdgcn_readlane(upto, 63);
        if (slot < all) {
            const int b = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto > slot));
            begin = __builtin_amdgcn_readlane(lo, b);
            len = __builtin_amdgcn_readlane(n, b);
            at = __builtin_amdgcn_readlane(upto, b) - 1 - slot;
            return true;
        }
        slot -= all;
    }
    return false;
}

// Workgroup -> slot and unit (a head, or a part of a group).  Workgroups go round-robin over the 8 XCDs; where units divide among them, neighbouring
// ones, which read the same keys and values, share an XCD and its L2.
__device__ __forceinline__ void slot_of(int bid, int units, int& slot, int& unit) {
    if (units & 7) {
        slot = bid / units;
        unit = bid % units;
    } else {
        const int per = units >> 3, j = bid >> 3;
        slot = j / per;
        unit = (bid & 7) * per + j % per;
    }
}

// ------------------------------------------------------------------ bf16 forward
template <int D, bool CAUSAL>
__global__ __launch_bounds__(NT) void packed_fwd_kernel(PackedArgs a) {
    constexpr int KS = D / 16, OT = D / 32;
    __shared__ __attribute__((aligned(16))) bf16_t Ks[2][64 * D];
    __shared__ __attribute__((aligned(16))) bf16_t Vs[2][64 * D];
    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, g = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int slot, h, begin, S, at;
    slot_of((int)blockIdx.x, a.heads, slot, h);
    if (!packed_tile<128, CAUSAL>(a.offsets, a.seqs, a.tokens, slot, lane, begin, S, at)) return;
    const int q0 = at * 128, d = a.d;
    const bf16_t* Qg = (const bf16_t*)a.q + (size_t)begin * a.ldq + h * d;
    const bf16_t* Kg = (const bf16_t*)a.k + (size_t)begin * a.ldk + h / a.group * d;
    const bf16_t* Vg = (const bf16_t*)a.v + (size_t)begin * a.ldv + h / a.group * d;
    const float scale_log2e = a.scale * LOG2E;
    const int wq0 = q0 + wave * 32, qrow = wq0 + l32;
    const unsigned ks0 = lds_address(Ks), vs0 = lds_address(Vs);
    constexpr unsigned TILE_BYTES = 64 * D * 2;

    const int kv_end = CAUSAL ? min(S, q0 + 128) : S;
    const int ntiles = (kv_end + 63) / 64;
    dma_utile<D>(Kg, a.ldk, 0, S - 1, d, ks0, wave, lane);
    dma_utile<D>(Vg, a.ldv, 0, S - 1, d, vs0, wave, lane);

    bf16x8 qf[KS];
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) qf[kk] = load_frag(Qg + (size_t)qrow * a.ldq + kk * 16 + g * 8, qrow < S && kk * 16 + g * 8 < d);

    f32x16 o[OT];
#pragma unroll
    for (int t = 0; t < OT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[t][r] = 0.f;
    float m = NEG_BIG, lsum = 0.f;          // lsum: over this lane's half of the keys

    auto step = [&](int t, auto buf_c) {        // LDS buffer index at compile time: addresses become base + immediate
        constexpr int buf = decltype(buf_c)::value;
        const int k0 = t * 64;
        wait_vmcnt<0>();                   // this wavefront's share of tile t has landed
        __syncthreads();                   // everyone's has; and tile t-1 is consumed, so its buffer is free
        if (t + 1 < ntiles) {
            dma_utile<D>(Kg, a.ldk, k0 + 64, S - 1, d, ks0 + (buf ^ 1) * TILE_BYTES, wave, lane);
            dma_utile<D>(Vg, a.ldv, k0 + 64, S - 1, d, vs0 + (buf ^ 1) * TILE_BYTES, wave, lane);
        }
        if (wq0 >= S || (CAUSAL && k0 > wq0 + 31)) return;           // wavefront-uniform: no query, or none that sees a key
        f32x16 s[2];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[kt][r] = 0.f;
#pragma unroll
            for (int kk = 0; kk < KS; ++kk)
                s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_us<D>(Ks[buf], kt * 32 + l32, kk, g), qf[kk], s[kt], 0, 0, 0);
        }
        // only tiles that reach past the sequence or the diagonal mask key by key (wavefront-uniform branch)
        if ((k0 + 63 >= S) || (CAUSAL && k0 + 63 > wq0)) {
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int key = k0 + kt * 32 + 8 * (r >> 2) + 4 * g + (r & 3);
                    if (key >= S || (CAUSAL && key > qrow)) s[kt][r] = NEG_BIG;
                }
        }
        // running maximum in the scaled (log2) domain; the scale is positive, so it commutes with max
        float mx = NEG_BIG;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[kt][r]);
        const float m_new = fmaxf(m, max32(mx) * scale_log2e);
        float rs = 0.f;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                // hardware exp2: arguments are <= 0 here, and flushing tiny results to zero is harmless
                const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kt][r], scale_log2e, -m_new));
                s[kt][r] = p;
                rs += p;
            }
        if (__builtin_amdgcn_ballot_w64(m_new != m)) {                  // the accumulators are rescaled where some row's maximum moved
            const float alpha = __builtin_amdgcn_exp2f(m - m_new);
            lsum *= alpha;
#pragma unroll
            for (int t2 = 0; t2 < OT; ++t2)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[t2][r] *= alpha;
        }
        lsum += rs;
        m = m_new;
#pragma unroll
        for (int J = 0; J < 4; ++J) {
            const bf16x8 pf = pack8(s[J >> 1], (J & 1) * 8);
#pragma unroll
            for (int t2 = 0; t2 < OT; ++t2)
                o[t2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_ut<D>(Vs[buf], t2 * 32, J, lane), pf, o[t2], 0, 0, 0);
        }
    };
    for (int t = 0; t < ntiles; t += 2) {
        step(t, std::integral_constant<int, 0>{});
        if (t + 1 < ntiles) step(t + 1, std::integral_constant<int, 1>{});
    }

    lsum = sum32(lsum);
    if (qrow < S) {
        const float inv = 1.0f / lsum;
        bf16_t* out = (bf16_t*)a.ctx + (size_t)(begin + qrow) * a.ldctx + h * d;
#pragma unroll
        for (int t2 = 0; t2 < OT; ++t2)
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4) {
                bf16x4 v;
#pragma unroll
                for (int c = 0; c < 4; ++c) v[c] = (bf16_t)(o[t2][r4 * 4 + c] * inv);
                if (t2 * 32 + 8 * r4 < d) *reinterpret_cast<bf16x4*>(out + t2 * 32 + 8 * r4 + 4 * g) = v;
            }
        if (g == 0) a.lse[(size_t)h * a.tokens + begin + qrow] = (m + log2f(lsum)) * LN2;
    }
}

// ----------------------------------------------------------------- bf16 backward
// LDS of one workgroup: two tensors x two stages of [64][D] tiles, and (dK/dV) the statistics of a tile's 64 queries.
template <int D> struct PackedBwdLds {
    bf16_t t0[2][64 * D], t1[2][64 * D];
    float lse2[2][64], dl[2][64];
};

// dQ of 128 queries (32 per wavefront), looping over 64-key tiles; forms delta of its queries and leaves it for the dK/dV kernel.
//   S^T = K Q^T (keys x queries)   P = exp2(S^T c - lse2)   dP^T = V dO^T
//   dS^T = P (dP^T - delta)        dQ^T += K^T dS^T (then * scale)
template <int D, bool CAUSAL>
__global__ __launch_bounds__(NT) void packed_dq_kernel(PackedArgs a) {
    constexpr int KS = D / 16, OT = D / 32;
    constexpr unsigned TILE_BYTES = 64 * D * 2;
    __shared__ __attribute__((aligned(16))) PackedBwdLds<D> sm;
    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, g = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int slot, h, begin, S, at;
    slot_of((int)blockIdx.x, a.heads, slot, h);
    if (!packed_tile<128, CAUSAL>(a.offsets, a.seqs, a.tokens, slot, lane, begin, S, at)) return;
    const int q0 = at * 128, d = a.d;
    const bf16_t* Qg = (const bf16_t*)a.q + (size_t)begin * a.ldq + h * d;
    const bf16_t* Kg = (const bf16_t*)a.k + (size_t)begin * a.ldk + h / a.group * d;
    const bf16_t* Vg = (const bf16_t*)a.v + (size_t)begin * a.ldv + h / a.group * d;
    const bf16_t* Og = (const bf16_t*)a.ctx + (size_t)begin * a.ldctx + h * d;
    const bf16_t* dOg = (const bf16_t*)a.dctx + (size_t)begin * a.lddctx + h * d;
    const size_t stat0 = (size_t)h * a.tokens + begin;
    const int wq0 = q0 + wave * 32, qrow = wq0 + l32;
    const float c2 = a.scale * LOG2E;
    const unsigned ks0 = lds_address(sm.t0), vs0 = lds_address(sm.t1);

    const int kv_end = CAUSAL ? min(S, q0 + 128) : S;
    const int ntiles = (kv_end + 63) / 64;
    auto fetch = [&](int t, int buf) {
        dma_utile<D>(Kg, a.ldk, t * 64, S - 1, d, ks0 + buf * TILE_BYTES, wave, lane);
        dma_utile<D>(Vg, a.ldv, t * 64, S - 1, d, vs0 + buf * TILE_BYTES, wave, lane);
    };
    fetch(0, 0);

    bf16x8 qf[KS], of[KS];
    float my_dl = 0.f;
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) {
        const bool ok = qrow < S && kk * 16 + g * 8 < d;
        qf[kk] = load_frag(Qg + (size_t)qrow * a.ldq + kk * 16 + g * 8, ok);
        of[kk] = load_frag(dOg + (size_t)qrow * a.lddctx + kk * 16 + g * 8, ok);
        const bf16x8 cf = load_frag(Og + (size_t)qrow * a.ldctx + kk * 16 + g * 8, ok);
#pragma unroll
        for (int e = 0; e < 8; ++e) my_dl += (float)of[kk][e] * (float)cf[e];
    }
    const float my_lse2 = qrow < S ? a.lse[stat0 + qrow] * LOG2E : 0.f;
    my_dl = sum32(my_dl);                                   // lanes l and l ^ 32 hold the whole row
    if (g == 0 && qrow < S) a.delta[stat0 + qrow] = my_dl;
    f32x16 dq[OT];
#pragma unroll
    for (int t = 0; t < OT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) dq[t][r] = 0.f;

    auto step = [&](int t, auto buf_c) {
        constexpr int buf = decltype(buf_c)::value;
        const int k0 = t * 64;
        wait_vmcnt<0>();
        __syncthreads();
        if (t + 1 < ntiles) fetch(t + 1, buf ^ 1);
        const bf16_t* Kt = sm.t0[buf];
        const bf16_t* Vt = sm.t1[buf];
        if (wq0 >= S || (CAUSAL && k0 > wq0 + 31)) return;
        const bool edge = (k0 + 63 >= S) || (CAUSAL && k0 + 63 > wq0);
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            f32x16 p, dp;
            // (at head dim 64 sixteen registers of -delta would cost the third wavefront per SIMD)
#pragma unroll
            for (int r = 0; r < 16; ++r) { p[r] = 0.f; dp[r] = D > 64 ? -my_dl : 0.f; }
#pragma unroll
            for (int kk = 0; kk < KS; ++kk) {
                p = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_us<D>(Kt, kt * 32 + l32, kk, g), qf[kk], p, 0, 0, 0);
                dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_us<D>(Vt, kt * 32 + l32, kk, g), of[kk], dp, 0, 0, 0);
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) p[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[r], c2, -my_lse2));
            if (edge) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int key = k0 + kt * 32 + 8 * (r >> 2) + 4 * g + (r & 3);
                    if (key >= S || (CAUSAL && key > qrow)) p[r] = 0.f;
                }
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) dp[r] = p[r] * (D > 64 ? dp[r] : dp[r] - my_dl);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const bf16x8 dsf = pack8(dp, j * 8);
#pragma unroll
                for (int t2 = 0; t2 < OT; ++t2)
                    dq[t2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_ut<D>(Kt, t2 * 32, kt * 2 + j, lane), dsf, dq[t2], 0, 0, 0);
            }
        }
    };
    for (int t = 0; t < ntiles; t += 2) {
        step(t, std::integral_constant<int, 0>{});
        if (t + 1 < ntiles) step(t + 1, std::integral_constant<int, 1>{});
    }
    if (qrow < S) {
        bf16_t* out = (bf16_t*)a.dq + (size_t)(begin + qrow) * a.lddq + h * d;
#pragma unroll
        for (int t2 = 0; t2 < OT; ++t2)
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4) {
                bf16x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = (bf16_t)(dq[t2][r4 * 4 + e] * a.scale);
                if (t2 * 32 + 8 * r4 < d) *reinterpret_cast<bf16x4*>(out + t2 * 32 + 8 * r4 + 4 * g) = v;
            }
    }
}

// dK, dV of 128 keys (32 per wavefront), looping over the heads of the group (of this workgroup's part of it) and, in each, over 64-query tiles.
//   S = Q K^T (queries x keys)   P = exp2(S c - lse2)     dP = dO V^T, started at -delta
//   dS = P dP                    dV^T += dO^T P           dK^T += Q^T dS (then * scale)
template <int D, bool CAUSAL>
__global__ __launch_bounds__(NT) void packed_dkv_kernel(PackedArgs a) {
    constexpr int KS = D / 16, OT = D / 32;
    constexpr unsigned TILE_BYTES = 64 * D * 2;
    __shared__ __attribute__((aligned(16))) PackedBwdLds<D> sm;
    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, g = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int slot, unit, begin, S, at;
    slot_of((int)blockIdx.x, a.kv_heads * a.splits, slot, unit);
    if (!packed_tile<128, CAUSAL>(a.offsets, a.seqs, a.tokens, slot, lane, begin, S, at)) return;
    const int kvh = unit / a.splits, part = unit % a.splits, d = a.d;
    const int h0 = kvh * a.group + part * (a.group / a.splits), hn = a.group / a.splits;
    const int j0 = ((S + 127) / 128 - 1 - at) * 128;        // the first keys meet the most queries
    const bf16_t* Kg = (const bf16_t*)a.k + (size_t)begin * a.ldk + kvh * d;
    const bf16_t* Vg = (const bf16_t*)a.v + (size_t)begin * a.ldv + kvh * d;
    const bf16_t* Qg = (const bf16_t*)a.q + (size_t)begin * a.ldq + h0 * d;
    const bf16_t* dOg = (const bf16_t*)a.dctx + (size_t)begin * a.lddctx + h0 * d;
    const float* lse = a.lse + (size_t)h0 * a.tokens + begin;
    const float* delta = a.delta + (size_t)h0 * a.tokens + begin;
    const int wj0 = j0 + wave * 32, jrow = wj0 + l32;
    const float c2 = a.scale * LOG2E;
    const unsigned qs0 = lds_address(sm.t0), os0 = lds_address(sm.t1);

    const int qt0 = CAUSAL ? j0 / 64 : 0;
    const int qtn = (S + 63) / 64, steps = (qtn - qt0) * hn;
    float stat = 0.f;                      // lse (threads 0..63) or -delta (threads 64..127) of the next tile
    int next_t = qt0, next_h = 0;          // the tile to be fetched
    auto fetch = [&](int buf) {
        const int i0 = next_t * 64;
        dma_utile<D>(Qg + next_h * d, a.ldq, i0, S - 1, d, qs0 + buf * TILE_BYTES, wave, lane);
        dma_utile<D>(dOg + next_h * d, a.lddctx, i0, S - 1, d, os0 + buf * TILE_BYTES, wave, lane);
        if (tid < 128) {
            const int i = i0 + (tid & 63);
            const size_t s = (size_t)next_h * a.tokens + i;
            stat = i < S ? (tid < 64 ? lse[s] * LOG2E : -delta[s]) : 0.f;
        }
        if (++next_t == qtn) { next_t = qt0; ++next_h; }
    };
    fetch(0);

    bf16x8 kf[KS], vf[KS];
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) {
        const bool ok = jrow < S && kk * 16 + g * 8 < d;
        kf[kk] = load_frag(Kg + (size_t)jrow * a.ldk + kk * 16 + g * 8, ok);
        vf[kk] = load_frag(Vg + (size_t)jrow * a.ldv + kk * 16 + g * 8, ok);
    }
    f32x16 dk[OT], dv[OT];
#pragma unroll
    for (int t = 0; t < OT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) { dk[t][r] = 0.f; dv[t][r] = 0.f; }

    int t = qt0;                           // the tile of the step
    auto step = [&](int i, auto buf_c) {
        constexpr int buf = decltype(buf_c)::value;
        const int i0 = t * 64;
        if (++t == qtn) t = qt0;
        wait_vmcnt<0>();                   // this wavefront's share of the tile (and its statistics) has arrived
        if (tid < 64) sm.lse2[buf][tid] = stat;
        else if (tid < 128) sm.dl[buf][tid - 64] = stat;
        __syncthreads();                   // the tile is complete in LDS; the one before is consumed by everyone
        if (i + 1 < steps) fetch(buf ^ 1);
        const bf16_t* Qt = sm.t0[buf];
        const bf16_t* Ot = sm.t1[buf];
        if (wj0 >= S || (CAUSAL && i0 + 63 < wj0)) return;           // wavefront-uniform: no key, or none that some query sees
        const bool edge = (i0 + 63 >= S) || (CAUSAL && i0 < wj0 + 31);
#pragma unroll
        for (int it = 0; it < 2; ++it) {
            f32x16 p, dp;
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4) {                       // 4 consecutive queries; dP starts at -delta
                const float4 d4 = *reinterpret_cast<const float4*>(&sm.dl[buf][it * 32 + 8 * r4 + 4 * g]);
                const float dv4[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
                for (int c = 0; c < 4; ++c) { p[r4 * 4 + c] = 0.f; dp[r4 * 4 + c] = dv4[c]; }
            }
#pragma unroll
            for (int kk = 0; kk < KS; ++kk) {
                p = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_us<D>(Qt, it * 32 + l32, kk, g), kf[kk], p, 0, 0, 0);
                dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_us<D>(Ot, it * 32 + l32, kk, g), vf[kk], dp, 0, 0, 0);
            }
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4) {
                const float4 l4 = *reinterpret_cast<const float4*>(&sm.lse2[buf][it * 32 + 8 * r4 + 4 * g]);
                const float lv[4] = {l4.x, l4.y, l4.z, l4.w};
#pragma unroll
                for (int c = 0; c < 4; ++c) p[r4 * 4 + c] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[r4 * 4 + c], c2, -lv[c]));
            }
            if (edge) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int q = i0 + it * 32 + 8 * (r >> 2) + 4 * g + (r & 3);
                    if (q >= S || (CAUSAL && q < jrow)) p[r] = 0.f;
                }
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) dp[r] *= p[r];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int J = it * 2 + j;
                const bf16x8 pf = pack8(p, j * 8);
                const bf16x8 dsf = pack8(dp, j * 8);
#pragma unroll
                for (int t2 = 0; t2 < OT; ++t2) {
                    dv[t2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_ut<D>(Ot, t2 * 32, J, lane), pf, dv[t2], 0, 0, 0);
                    dk[t2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_ut<D>(Qt, t2 * 32, J, lane), dsf, dk[t2], 0, 0, 0);
                }
            }
        }
    };
    for (int i = 0; i < steps; i += 2) {
        step(i, std::integral_constant<int, 0>{});
        if (i + 1 < steps) step(i + 1, std::integral_constant<int, 1>{});
    }
    if (jrow >= S) return;
    const size_t row = (size_t)(begin + jrow);
    if (a.splits > 1) {
        const size_t width = (size_t)a.kv_heads * d, slab = (size_t)a.tokens * width;
        float* out = a.slabs + (size_t)part * 2 * slab + row * width + kvh * d;
#pragma unroll
        for (int t2 = 0; t2 < OT; ++t2)
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4) {
                f32x4 x, y;
#pragma unroll
                for (int e = 0; e < 4; ++e) { x[e] = dk[t2][r4 * 4 + e] * a.scale; y[e] = dv[t2][r4 * 4 + e]; }
                if (t2 * 32 + 8 * r4 >= d) continue;
                *reinterpret_cast<f32x4*>(out + t2 * 32 + 8 * r4 + 4 * g) = x;
                *reinterpret_cast<f32x4*>(out + slab + t2 * 32 + 8 * r4 + 4 * g) = y;
            }
        return;
    }
    bf16_t* dko = (bf16_t*)a.dk + row * a.lddk + kvh * d;
    bf16_t* dvo = (bf16_t*)a.dv + row * a.lddv + kvh * d;
#pragma unroll
    for (int t2 = 0; t2 < OT; ++t2)
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
            bf16x4 x, y;
#pragma unroll
            for (int e = 0; e < 4; ++e) { x[e] = (bf16_t)(dk[t2][r4 * 4 + e] * a.scale); y[e] = (bf16_t)dv[t2][r4 * 4 + e]; }
            if (t2 * 32 + 8 * r4 >= d) continue;
            *reinterpret_cast<bf16x4*>(dko + t2 * 32 + 8 * r4 + 4 * g) = x;
            *reinterpret_cast<bf16x4*>(dvo + t2 * 32 + 8 * r4 + 4 * g) = y;
        }
}

// dk, dv = the sums of the parts' slabs, in the order of the parts, over the rows that sequences own.  A thread takes 4 columns of a row.
template <typename T>
__global__ __launch_bounds__(NT) void packed_join_kernel(PackedArgs a) {
    const int width = a.kv_heads * a.d, chunks = width / 4;
    const int first = min(max(a.offsets[0], 0), a.tokens), end = min(max(a.offsets[a.seqs], 0), a.tokens);
    const size_t slab = (size_t)a.tokens * width;
    for (size_t i = (size_t)blockIdx.x * NT + threadIdx.x; i < (size_t)a.tokens * chunks; i += (size_t)gridDim.x * NT) {
        const int row = (int)(i / chunks), c = (int)(i % chunks) * 4;
        if (row < first || row >= end) continue;
        const float* p = a.slabs + (size_t)row * width + c;
        f32x4 x = *reinterpret_cast<const f32x4*>(p), y = *reinterpret_cast<const f32x4*>(p + slab);
        for (int s = 1; s < a.splits; ++s) {
            x += *reinterpret_cast<const f32x4*>(p + (size_t)s * 2 * slab);
            y += *reinterpret_cast<const f32x4*>(p + (size_t)s * 2 * slab + slab);
        }
        T* dk = (T*)a.dk + (size_t)row * a.lddk + c;
        T* dv = (T*)a.dv + (size_t)row * a.lddv + c;
        typedef T vec4 __attribute__((ext_vector_type(4)));
        *reinterpret_cast<vec4*>(dk) = __builtin_convertvector(x, vec4);
        *reinterpret_cast<vec4*>(dv) = __builtin_convertvector(y, vec4);
    }
}

// ----------------------------------------------------------------- float forward
template <int D, bool CAUSAL>
__global__ __launch_bounds__(NT) void packed_fwd_f32_kernel(PackedArgs a) {
    constexpr int OT = D / 32;
    __shared__ float lds[NW * OT * 16 * WAVE];
    __shared__ float stat[2][NW][32];
    const int lane = threadIdx.x & 63, l32 = lane & 31, g = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int slot, h, begin, S, at;
    slot_of((int)blockIdx.x, a.heads, slot, h);
    if (!packed_tile<TILE, CAUSAL>(a.offsets, a.seqs, a.tokens, slot, lane, begin, S, at)) return;
    const int q0 = at * TILE, d = a.d;
    const float* Qg = (const float*)a.q + (size_t)begin * a.ldq + h * d;
    const float* Kg = (const float*)a.k + (size_t)begin * a.ldk + h / a.group * d;
    const float* Vg = (const float*)a.v + (size_t)begin * a.ldv + h / a.group * d;
    const float scale_log2e = a.scale * LOG2E;
    const int qrow = q0 + l32;
    RowFrag<D> q;
    q.load(Qg + (size_t)min(qrow, S - 1) * a.ldq, d, g, true);
    f32x16 o[OT];
#pragma unroll
    for (int t = 0; t < OT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[t][r] = 0.f;
    float m = NEG_BIG, lsum = 0.f;
    const int kend = CAUSAL ? min(S, q0 + TILE) : S;
    for (int k0 = wave * TILE; k0 < kend; k0 += NW * TILE) {
        RowFrag<D> k;
        ColFrag<D> v;
        k.load(Kg + (size_t)min(k0 + l32, S - 1) * a.ldk, d, g, false);
        v.load(Vg, a.ldv, k0, S - 1, d, l32, g);
        f32x16 s = dot_rows<D>(k, q);
        if (k0 + TILE > S || (CAUSAL && k0 + TILE - 1 > q0)) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int key = k0 + 8 * (r >> 2) + 4 * g + (r & 3);
                if (key >= S || (CAUSAL && key > qrow)) s[r] = NEG_BIG;
            }
        }
        float mx = s[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
        mx = max32(mx) * scale_log2e;
        const float m_new = fmaxf(m, mx), alpha = __builtin_amdgcn_exp2f(m - m_new);
        float rs = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], scale_log2e, -m_new));
            rs += s[r];
        }
        lsum = lsum * alpha + sum32(rs);
        m = m_new;
#pragma unroll
        for (int t = 0; t < OT; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[t][r] *= alpha;
        add_outer<D>(o, v, s);
    }
    // the wavefronts' partial softmaxes: common maximum, rescaled sums
    if (g == 0) { stat[0][wave][l32] = m; stat[1][wave][l32] = lsum; }
    __syncthreads();
    float M = stat[0][0][l32];
#pragma unroll
    for (int w = 1; w < NW; ++w) M = fmaxf(M, stat[0][w][l32]);
    float total = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) total += stat[1][w][l32] * __builtin_amdgcn_exp2f(stat[0][w][l32] - M);
    const float mine = __builtin_amdgcn_exp2f(m - M);           // 0 for a wavefront that saw no key
#pragma unroll
    for (int t = 0; t < OT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[t][r] *= mine;
    f32x4 out[OT];
    combine<D>(lds, o, out, wave, lane);
    if (qrow < S) {
        store_rows<D>((float*)a.ctx + (size_t)(begin + qrow) * a.ldctx + h * d, out, 1.0f / total, d, wave, g);
        if (wave == 0 && g == 0) a.lse[(size_t)h * a.tokens + begin + qrow] = __builtin_fmaf(M, LN2, __builtin_fmaf(M, LN2_LOW, logf(total)));
    }
}

// ---------------------------------------------------------------- float backward
// dQ of 32 queries; delta = rowsum(dO * O) of the queries on the way.
template <int D, bool CAUSAL>
__device__ __forceinline__ void packed_dq_f32(float* lds, int bid, const PackedArgs& a) {
    constexpr int OT = D / 32;
    const int lane = threadIdx.x & 63, l32 = lane & 31, g = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int slot, h, begin, S, at;
    slot_of(bid, a.heads, slot, h);
    if (!packed_tile<TILE, CAUSAL>(a.offsets, a.seqs, a.tokens, slot, lane, begin, S, at)) return;
    const int q0 = at * TILE, d = a.d;
    const float* Kg = (const float*)a.k + (size_t)begin * a.ldk + h / a.group * d;
    const float* Vg = (const float*)a.v + (size_t)begin * a.ldv + h / a.group * d;
    const int qrow = q0 + l32;
    const size_t qr = (size_t)begin + min(qrow, S - 1);
    RowFrag<D> q, dO, o;
    q.load((const float*)a.q + qr * a.ldq + h * d, d, g, true);
    dO.load((const float*)a.dctx + qr * a.lddctx + h * d, d, g, true);
    o.load((const float*)a.ctx + qr * a.ldctx + h * d, d, g, true);
    const float my_lse = a.lse[(size_t)h * a.tokens + qr];
    float delta = 0.f;
#pragma unroll
    for (int i = 0; i < D / 8; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) delta += dO.v[i][j] * o.v[i][j];
    delta = sum32(delta);
    f32x16 dq[OT];
#pragma unroll
    for (int t = 0; t < OT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) dq[t][r] = 0.f;
    const int kend = CAUSAL ? min(S, q0 + TILE) : S;
    for (int k0 = wave * TILE; k0 < kend; k0 += NW * TILE) {
        RowFrag<D> k, v;
        ColFrag<D> kt;
        const size_t kr = (size_t)min(k0 + l32, S - 1);
        k.load(Kg + kr * a.ldk, d, g, false);
        v.load(Vg + kr * a.ldv, d, g, false);
        kt.load(Kg, a.ldk, k0, S - 1, d, l32, g);
        f32x16 p = dot_rows<D>(k, q), dp = dot_rows<D>(v, dO);
#pragma unroll
        for (int r = 0; r < 16; ++r) p[r] = prob(p[r], a.scale, my_lse);
        if (k0 + TILE > S || (CAUSAL && k0 + TILE - 1 > q0)) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int key = k0 + 8 * (r >> 2) + 4 * g + (r & 3);
                if (key >= S || (CAUSAL && key > qrow)) p[r] = 0.f;
            }
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) dp[r] = p[r] * (dp[r] - delta);
        add_outer<D>(dq, kt, dp);
    }
    f32x4 out[OT];
    combine<D>(lds, dq, out, wave, lane);
    if (qrow < S) store_rows<D>((float*)a.dq + qr * a.lddq + h * d, out, a.scale, d, wave, g);
}

// dK, dV of 32 keys; the wavefronts deal the (head, tile of queries) pairs of the part among themselves.
template <int D, bool CAUSAL>
__device__ __forceinline__ void packed_dkv_f32(float* lds, int bid, const PackedArgs& a) {
    constexpr int OT = D / 32;
    const int lane = threadIdx.x & 63, l32 = lane & 31, g = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int slot, unit, begin, S, at;
    slot_of(bid, a.kv_heads * a.splits, slot, unit);
    if (!packed_tile<TILE, CAUSAL>(a.offsets, a.seqs, a.tokens, slot, lane, begin, S, at)) return;
    const int kvh = unit / a.splits, part = unit % a.splits, d = a.d;
    const int h0 = kvh * a.group + part * (a.group / a.splits), hn = a.group / a.splits;
    const int j0 = ((S + TILE - 1) / TILE - 1 - at) * TILE;          // the first keys meet the most queries
    const int jrow = j0 + l32;
    const size_t jr = (size_t)begin + min(jrow, S - 1);
    RowFrag<D> k, v;
    k.load((const float*)a.k + jr * a.ldk + kvh * d, d, g, true);
    v.load((const float*)a.v + jr * a.ldv + kvh * d, d, g, true);
    f32x16 dk[OT], dv[OT];
#pragma unroll
    for (int t = 0; t < OT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) { dk[t][r] = 0.f; dv[t][r] = 0.f; }
    const int first = CAUSAL ? j0 : 0, tiles = (S - first + TILE - 1) / TILE;
    int h = h0, i0 = first + wave * TILE;
    for (int n = wave; n < tiles * hn; n += NW, i0 += NW * TILE) {
        while (i0 >= first + tiles * TILE) { i0 -= tiles * TILE; ++h; }
        const int ir = min(i0 + l32, S - 1);
        const size_t qr = (size_t)begin + ir;
        RowFrag<D> q, dO, o;
        ColFrag<D> qt, dOt;
        q.load((const float*)a.q + qr * a.ldq + h * d, d, g, false);
        dO.load((const float*)a.dctx + qr * a.lddctx + h * d, d, g, true);
        o.load((const float*)a.ctx + qr * a.ldctx + h * d, d, g, true);
        dOt.load((const float*)a.dctx + (size_t)begin * a.lddctx + h * d, a.lddctx, i0, S - 1, d, l32, g);
        qt.load((const float*)a.q + (size_t)begin * a.ldq + h * d, a.ldq, i0, S - 1, d, l32, g);
        const float my_lse = a.lse[(size_t)h * a.tokens + qr];
        float delta = 0.f;                       // of row l32; the rows of the score registers fetch theirs from its lane
#pragma unroll
        for (int i = 0; i < D / 8; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) delta += dO.v[i][j] * o.v[i][j];
        delta = sum32(delta);
        f32x16 p = dot_rows<D>(q, k), dp = dot_rows<D>(dO, v);
        const bool edge = i0 + TILE > S || (CAUSAL && i0 < j0 + TILE - 1);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int ii = 8 * (r >> 2) + 4 * g + (r & 3);
            p[r] = prob(p[r], a.scale, __shfl(my_lse, ii, WAVE));
            if (edge && (i0 + ii >= S || (CAUSAL && i0 + ii < jrow))) p[r] = 0.f;
            dp[r] = p[r] * (dp[r] - __shfl(delta, ii, WAVE));
        }
        add_outer<D>(dv, dOt, p);
        add_outer<D>(dk, qt, dp);
    }
    const size_t width = (size_t)a.kv_heads * d, slab = (size_t)a.tokens * width;
    float* dko = a.splits > 1 ? a.slabs + (size_t)part * 2 * slab + jr * width + kvh * d : (float*)a.dk + jr * a.lddk + kvh * d;
    float* dvo = a.splits > 1 ? a.slabs + (size_t)part * 2 * slab + slab + jr * width + kvh * d : (float*)a.dv + jr * a.lddv + kvh * d;
    f32x4 out[OT];
    combine<D>(lds, dv, out, wave, lane);
    if (jrow < S) store_rows<D>(dvo, out, 1.0f, d, wave, g);
    __syncthreads();                             // everyone has read the dV sums
    combine<D>(lds, dk, out, wave, lane);
    if (jrow < S) store_rows<D>(dko, out, a.scale, d, wave, g);
}

// Both roles in one launch, the longer one first; each forms the delta it needs.
template <int D, bool CAUSAL>
__global__ __launch_bounds__(NT) void packed_bwd_f32_kernel(PackedArgs a, int dkv) {
    __shared__ float lds[NW * (D / 32) * 16 * WAVE];
    const int bid = (int)blockIdx.x;
    if (bid < dkv) packed_dkv_f32<D, CAUSAL>(lds, bid, a);
    else packed_dq_f32<D, CAUSAL>(lds, bid - dkv, a);
}

// ------------------------------------------------------------------------- host
int tile_rows(int dtype) { return dtype == CHIMERA_F32 ? TILE : 128; }

// Slots for every tile that `tokens` rows in `seqs` sequences can have: a full one for each tile's rows, one more that is not full for each sequence
size_t slots(int dtype, int seqs, int tokens) { return (size_t)tokens / tile_rows(dtype) + (size_t)std::min(seqs, tokens); }

// Parts of a group's heads: the fewest that give dK and dV 600 workgroups
int group_parts(int dtype, int tokens, int kv_heads, int group) {
    const size_t some = (size_t)kv_heads * ((tokens + tile_rows(dtype) - 1) / tile_rows(dtype));
    for (int s = 1; s < group; ++s)
        if (group % s == 0 && some * s >= 600) return s;
    return group;
}

struct BwdLayout { size_t delta, slabs, total; int splits; };
BwdLayout bwd_layout(int dtype, int tokens, int heads, int kv_heads, int d) {
    BwdLayout l{};
    l.splits = group_parts(dtype, tokens, kv_heads, heads / kv_heads);
    l.slabs = ((size_t)heads * tokens * 4 + 255) & ~(size_t)255;
    l.total = l.slabs + (l.splits > 1 ? (size_t)l.splits * 2 * tokens * kv_heads * d * 4 : 0);
    return l;
}

int check_packed(int dtype, int seqs, int tokens, int heads, int kv_heads, int d) {
    if (dtype != CHIMERA_F32 && dtype != CHIMERA_BF16) return fail(CHIMERA_EINVAL, "unknown dtype %d", dtype);
    if (seqs < 1 || tokens < 1 || heads < 1 || kv_heads < 1) return fail(CHIMERA_EINVAL, "sizes must be positive");
    if (heads % kv_heads) return fail(CHIMERA_EINVAL, "heads=%d must be a multiple of kv_heads=%d", heads, kv_heads);
    const int unit = dtype == CHIMERA_F32 ? 4 : 8;
    if (d < unit || d > 128 || d % unit) return fail(CHIMERA_EINVAL, "head_dim=%d must be a multiple of %d up to 128", d, unit);
    if ((long)heads * d > 1 << 16) return fail(CHIMERA_EINVAL, "more than 2^16 columns of query heads");
    if (tokens > 1 << 28 || seqs > 1 << 28 || (size_t)heads * (slots(dtype, seqs, tokens) + 8) >= (size_t)1 << 30)
        return fail(CHIMERA_EINVAL, "more than 2^28 tokens, or 2^30 tiles of all heads");
    return CHIMERA_OK;
}

int check_rows(const char* what, const void* p, int ld, int cols, int dtype) {
    const int unit = dtype == CHIMERA_F32 ? 4 : 8;
    if (!p) return fail(CHIMERA_EINVAL, "%s is NULL", what);
    if (ld < cols || ld % unit) return fail(CHIMERA_EINVAL, "rows of %s are %d apart: a multiple of %d and at least %d expected", what, ld, unit, cols);
    if ((uintptr_t)p & 15) return fail(CHIMERA_EINVAL, "%s must be 16-byte aligned", what);
    return CHIMERA_OK;
}

#define PACKED_TRY(expr) do { int rc__ = (expr); if (rc__) return rc__; } while (0)
#define PACKED_GO(KERNEL, D, GRID, ...)                                                                              \
    do {                                                                                                             \
        if (causal) hipLaunchKernelGGL((KERNEL<D, true>), dim3((unsigned)(GRID)), dim3(NT), 0, s, __VA_ARGS__);       \
        else hipLaunchKernelGGL((KERNEL<D, false>), dim3((unsigned)(GRID)), dim3(NT), 0, s, __VA_ARGS__);             \
        CHIMERA_LAUNCH_CHECK("attention over packed sequences");                                                     \
    } while (0)

}  // namespace

}  // namespace chimera

using namespace chimera;

extern "C" {

size_t chimera_op_attention_packed_bwd_workspace_bytes(int dtype, int seqs, int tokens, int heads, int kv_heads, int head_dim) {
    return check_packed(dtype, seqs, tokens, heads, kv_heads, head_dim) ? 0 : bwd_layout(dtype, tokens, heads, kv_heads, head_dim).total;
}

int chimera_op_attention_packed_fwd(int dtype, int seqs, int tokens, int heads, int kv_heads, int head_dim, int causal, float scale,
                                    const int32_t* d_offsets, const void* d_q, int ldq, const void* d_k, int ldk, const void* d_v, int ldv,
                                    void* d_ctx, int ldctx, float* d_lse, void* hip_stream) {
    PACKED_TRY(check_packed(dtype, seqs, tokens, heads, kv_heads, head_dim));
    if (!(scale > 0) || scale > 3e38f) return fail(CHIMERA_EINVAL, "scale must be positive and finite");
    if (!d_offsets || !d_lse || (((uintptr_t)d_offsets | (uintptr_t)d_lse) & 3)) return fail(CHIMERA_EINVAL, "offsets or lse is NULL or not aligned");
    const int wide = heads * head_dim, narrow = kv_heads * head_dim;
    PACKED_TRY(check_rows("q", d_q, ldq, wide, dtype));
    PACKED_TRY(check_rows("k", d_k, ldk, narrow, dtype));
    PACKED_TRY(check_rows("v", d_v, ldv, narrow, dtype));
    PACKED_TRY(check_rows("ctx", d_ctx, ldctx, wide, dtype));
    const size_t e = dtype == CHIMERA_F32 ? 4 : 2, n = (size_t)tokens;
    PACKED_TRY(check_apart({matrix(d_q, n, wide, ldq, e), matrix(d_k, n, narrow, ldk, e), matrix(d_v, n, narrow, ldv, e), plain(d_offsets, ((size_t)seqs + 1) * 4)},
                           {matrix(d_ctx, n, wide, ldctx, e), plain(d_lse, n * heads * 4)}));
    PackedArgs a{};
    a.offsets = d_offsets; a.seqs = seqs; a.tokens = tokens; a.heads = heads; a.kv_heads = kv_heads; a.group = heads / kv_heads; a.d = head_dim; a.scale = scale;
    a.q = d_q; a.k = d_k; a.v = d_v; a.ldq = ldq; a.ldk = ldk; a.ldv = ldv; a.ctx = d_ctx; a.ldctx = ldctx; a.lse = d_lse;
    hipStream_t s = (hipStream_t)hip_stream;
    const size_t grid = slots(dtype, seqs, tokens) * heads;
    if (dtype == CHIMERA_F32) {
        if (head_dim <= 32) PACKED_GO(packed_fwd_f32_kernel, 32, grid, a);
        else if (head_dim <= 64) PACKED_GO(packed_fwd_f32_kernel, 64, grid, a);
        else PACKED_GO(packed_fwd_f32_kernel, 128, grid, a);
    } else {
        if (head_dim <= 64) PACKED_GO(packed_fwd_kernel, 64, grid, a);
        else PACKED_GO(packed_fwd_kernel, 128, grid, a);
    }
    return CHIMERA_OK;
}

int chimera_op_attention_packed_bwd(int dtype, int seqs, int tokens, int heads, int kv_heads, int head_dim, int causal, float scale,
                                    const int32_t* d_offsets, const void* d_q, int ldq, const void* d_k, int ldk, const void* d_v, int ldv,
                                    const void* d_ctx, int ldctx, const float* d_lse, const void* d_dctx, int lddctx, void* d_dq, int lddq,
                                    void* d_dk, int lddk, void* d_dv, int lddv, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
    PACKED_TRY(check_packed(dtype, seqs, tokens, heads, kv_heads, head_dim));
    if (!(scale > 0) || scale > 3e38f) return fail(CHIMERA_EINVAL, "scale must be positive and finite");
    if (!d_offsets || !d_lse || (((uintptr_t)d_offsets | (uintptr_t)d_lse) & 3)) return fail(CHIMERA_EINVAL, "offsets or lse is NULL or not aligned");
    const int wide = heads * head_dim, narrow = kv_heads * head_dim;
    PACKED_TRY(check_rows("q", d_q, ldq, wide, dtype));
    PACKED_TRY(check_rows("k", d_k, ldk, narrow, dtype));
    PACKED_TRY(check_rows("v", d_v, ldv, narrow, dtype));
    PACKED_TRY(check_rows("ctx", d_ctx, ldctx, wide, dtype));
    PACKED_TRY(check_rows("dctx", d_dctx, lddctx, wide, dtype));
    PACKED_TRY(check_rows("dq", d_dq, lddq, wide, dtype));
    PACKED_TRY(check_rows("dk", d_dk, lddk, narrow, dtype));
    PACKED_TRY(check_rows("dv", d_dv, lddv, narrow, dtype));
    if (!d_workspace || ((uintptr_t)d_workspace & 255)) return fail(CHIMERA_EINVAL, "workspace is NULL or not 256-byte aligned");
    const BwdLayout l = bwd_layout(dtype, tokens, heads, kv_heads, head_dim);
    if (workspace_bytes < l.total) return fail(CHIMERA_ENOMEM, "workspace holds %zu bytes, need %zu", workspace_bytes, l.total);
    const size_t e = dtype == CHIMERA_F32 ? 4 : 2, n = (size_t)tokens;
    PACKED_TRY(check_apart({matrix(d_q, n, wide, ldq, e), matrix(d_k, n, narrow, ldk, e), matrix(d_v, n, narrow, ldv, e), matrix(d_ctx, n, wide, ldctx, e),
                            matrix(d_dctx, n, wide, lddctx, e), plain(d_lse, n * heads * 4), plain(d_offsets, ((size_t)seqs + 1) * 4)},
                           {matrix(d_dq, n, wide, lddq, e), matrix(d_dk, n, narrow, lddk, e), matrix(d_dv, n, narrow, lddv, e), plain(d_workspace, l.total)}));
    PackedArgs a{};
    a.offsets = d_offsets; a.seqs = seqs; a.tokens = tokens; a.heads = heads; a.kv_heads = kv_heads; a.group = heads / kv_heads; a.d = head_dim; a.scale = scale;
    a.q = d_q; a.k = d_k; a.v = d_v; a.ldq = ldq; a.ldk = ldk; a.ldv = ldv; a.ctx = (void*)d_ctx; a.ldctx = ldctx; a.lse = (float*)d_lse;
    a.dctx = d_dctx; a.lddctx = lddctx; a.dq = d_dq; a.dk = d_dk; a.dv = d_dv; a.lddq = lddq; a.lddk = lddk; a.lddv = lddv;
    a.delta = (float*)d_workspace; a.slabs = (float*)((char*)d_workspace + l.slabs); a.splits = l.splits;
    hipStream_t s = (hipStream_t)hip_stream;
    const size_t dq_grid = slots(dtype, seqs, tokens) * heads, dkv_grid = slots(dtype, seqs, tokens) * kv_heads * l.splits;
    if (dtype == CHIMERA_F32) {
        if (head_dim <= 32) PACKED_GO(packed_bwd_f32_kernel, 32, dq_grid + dkv_grid, a, (int)dkv_grid);
        else if (head_dim <= 64) PACKED_GO(packed_bwd_f32_kernel, 64, dq_grid + dkv_grid, a, (int)dkv_grid);
        else PACKED_GO(packed_bwd_f32_kernel, 128, dq_grid + dkv_grid, a, (int)dkv_grid);
    } else if (head_dim <= 64) {
        PACKED_GO(packed_dq_kernel, 64, dq_grid, a);
        PACKED_GO(packed_dkv_kernel, 64, dkv_grid, a);
    } else {
        PACKED_GO(packed_dq_kernel, 128, dq_grid, a);
        PACKED_GO(packed_dkv_kernel, 128, dkv_grid, a);
    }
    if (l.splits > 1) {
        const size_t chunks = (size_t)tokens * narrow / 4;
        const dim3 grid((unsigned)std::min<size_t>((chunks + NT - 1) / NT, 4096));
        if (dtype == CHIMERA_F32) hipLaunchKernelGGL(packed_join_kernel<float>, grid, dim3(NT), 0, s, a);
        else hipLaunchKernelGGL(packed_join_kernel<bf16_t>, grid, dim3(NT), 0, s, a);
        CHIMERA_LAUNCH_CHECK("attention over packed sequences");
    }
    return CHIMERA_OK;
}

}  // extern "C"
