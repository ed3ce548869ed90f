// What joins a branch of a block to the residual stream, and its gradients:
//
//   u = N1(f),   y = alpha x + beta gate u,   h = N2(y),     N(v) = (v - mean) rstd gain + bias
//
// f is the branch's result, x the stream, y the stream behind the block, h the next branch's operand.  Each norm is none, LayerNorm or RMSNorm (mean 0), and the
// gate one row for every `run` consecutive rows, or none.  Backward, with n^ = (v - mean) rstd and s over a row's columns:
//
//   dy~ = dy + N2'(dh),   dx = alpha dy~,   du = beta gate dy~,   df = N1'(du),   N'(d) = rstd (d gain - s(d gain) / cols - n^ s(d gain n^) / cols)
//   dgain2 = sum dh y^,   dbias2 = sum dh,   dgate = sum beta u dy~,   dgain1 = sum du f^,   dbias1 = sum du       (sums over rows)
//
// (an RMSNorm has no term s(d gain)).  Both directions are one pass over memory, which bounds them: a row stays in registers from its loads to its stores,
// 8 columns a thread and chunk, and 64 to 512 threads share it.
#include "device.h"
#include "spans.h"

#include <cmath>

namespace chimera {

namespace {

constexpr int V = 8;                     // columns of a chunk
constexpr int BN_COLS = 8192;
constexpr int ROW_GROUPS = 512;          // workgroups of the backward

// A chunk as it comes from memory
template <typename T> struct Chunk {
    uint4 q[V / Elem<T>::VEC];
    __device__ __forceinline__ void load(const T* p) {
#pragma unroll
        for (int i = 0; i < V / Elem<T>::VEC; ++i) q[i] = *reinterpret_cast<const uint4*>(p + i * Elem<T>::VEC);
    }
    __device__ __forceinline__ void unpack(float* out) const {
#pragma unroll
        for (int i = 0; i < V / Elem<T>::VEC; ++i) load_vec<T>(reinterpret_cast<const T*>(&q[i]), out + i * Elem<T>::VEC);
    }
};

// A chunk of the stream (y, dx), which is read again behind the next branch: stored past the caches' order of use, where its lines push out what is read sooner.  h and df are the next
// operator's operands and stay (8192 x 1600 bf16, norms and gate with the product behind them: all results past the caches 187 us, the stream 168, none 168; 8192 x 2048 with a float stream,
// the norms alone, 41.4, 41.6 and 44.2).
template <typename T> __device__ __forceinline__ void store_stream(T* p, const float* v) {
    typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int i = 0; i < V; i += Elem<T>::VEC) {
        T w[Elem<T>::VEC];
#pragma unroll
        for (int e = 0; e < Elem<T>::VEC; ++e) w[e] = Elem<T>::from_f(v[i + e]);
        u32x4 q;
        __builtin_memcpy(&q, w, sizeof(q));
        __builtin_nontemporal_store(q, reinterpret_cast<u32x4*>(p + i));
    }
}

struct JoinArgs {
    int rows, cols, run;                 // run: rows that share a row of the gate
    int post, pre;
    float eps, alpha, beta;
    const void *f, *x, *gate, *post_gain, *post_bias, *pre_gain, *pre_bias;
    void *y, *h;
    float* stats;                        // [4][rows]: mean and rstd of N1, of N2
    int per_group;                       // rows of a workgroup
    // backward
    const void *dy, *dh;
    void *dx, *df;
    int sums;                            // which column sums are wanted, bit by bit in the order of the slots
    int whole_runs;                      // dgate: a workgroup holds whole runs of the gate (else a run holds whole workgroups)
    int groups_per_run;
    float* partial;                      // [workgroups][slots][cols]; null: the sums are final
    float* out[5];
    int overwrite;
};
enum { SUM_GAIN1, SUM_BIAS1, SUM_GAIN2, SUM_BIAS2, SUM_GATE, SUMS };

// Sums of N numbers over the TPR threads that share a row; `lds` holds N floats for each wavefront of the workgroup.  Every thread of the workgroup comes here, and
// a call's `lds` is not used again by the next one: one barrier each is then enough.
template <int TPR, int N> __device__ __forceinline__ void row_sums(float (&v)[N], float* lds, int wave, int lane) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
    if constexpr (TPR > WAVE) {
        constexpr int PER = TPR / WAVE;
        if (lane == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) lds[wave * N + i] = v[i];
        __syncthreads();
        const int w0 = wave / PER * PER;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = lds[w0 * N + i];
#pragma unroll
            for (int w = 1; w < PER; ++w) v[i] += lds[(w0 + w) * N + i];
        }
    }
}

// ---------------------------------------------------------------------- forward
template <typename T, typename TS, int TPR, int MAXT>
__global__ __launch_bounds__(256) void join_fwd_kernel(JoinArgs a) {
    constexpr int LANES = 256 / TPR;                        // rows side by side
    __shared__ float lds[2][4][4];
    const int tid = threadIdx.x, lane = tid % WAVE, wave = tid / WAVE, c0 = tid % TPR, cols = a.cols, nchunk = cols / V;
    const float inv_cols = 1.0f / (float)cols;
    const int first = blockIdx.x * a.per_group, last = min(a.rows, first + a.per_group);
    for (int base = first, odd = 0; base < last; base += LANES, odd ^= 1) {    // the same count for every thread
        const int row = min(base + tid / TPR, last - 1);
        const bool mine = base + tid / TPR < last;
        const size_t at = (size_t)row * cols;
        Chunk<T> rf[MAXT];
        Chunk<TS> rx[MAXT];
#pragma unroll
        for (int t = 0; t < MAXT; ++t) {
            const size_t c = at + min(c0 + t * TPR, nchunk - 1) * V;
            rf[t].load((const T*)a.f + c);
            if (a.x) rx[t].load((const TS*)a.x + c);
        }
        float u[MAXT][V];
        float s[1] = {0.f};
#pragma unroll
        for (int t = 0; t < MAXT; ++t) rf[t].unpack(u[t]);
        if (a.post) {
            float mean = 0.f;
            if (a.post == CHIMERA_NORM_LAYER) {
#pragma unroll
                for (int t = 0; t < MAXT; ++t)
                    if (c0 + t * TPR < nchunk)
#pragma unroll
                        for (int e = 0; e < V; ++e) s[0] += u[t][e];
                row_sums<TPR>(s, lds[odd][0], wave, lane);
                mean = s[0] * inv_cols;
                s[0] = 0.f;
            }
#pragma unroll
            for (int t = 0; t < MAXT; ++t)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    u[t][e] -= mean;
                    if (c0 + t * TPR < nchunk) s[0] += u[t][e] * u[t][e];
                }
            row_sums<TPR>(s, lds[odd][1], wave, lane);
            const float rstd = 1.0f / sqrtf(s[0] * inv_cols + a.eps);
            if (mine && c0 == 0) { a.stats[row] = mean; a.stats[(size_t)a.rows + row] = rstd; }
#pragma unroll
            for (int t = 0; t < MAXT; ++t) {
                const int c = min(c0 + t * TPR, nchunk - 1) * V;
                float g[V], b[V];
                load_elems<T, V>((const T*)a.post_gain + c, g);
                if (a.post_bias) load_elems<T, V>((const T*)a.post_bias + c, b);
#pragma unroll
                for (int e = 0; e < V; ++e) u[t][e] = u[t][e] * rstd * g[e] + (a.post_bias ? b[e] : 0.f);
            }
        }
        const T* gate = a.gate ? (const T*)a.gate + (size_t)(row / a.run) * cols : nullptr;
        s[0] = 0.f;
#pragma unroll
        for (int t = 0; t < MAXT; ++t) {
            const int c = min(c0 + t * TPR, nchunk - 1) * V;
            float g[V], x[V];
            if (gate) load_elems<T, V>(gate + c, g);
            if (a.x) rx[t].unpack(x);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                u[t][e] *= gate ? a.beta * g[e] : a.beta;
                if (a.x) u[t][e] += a.alpha * x[e];
                if (c0 + t * TPR < nchunk) s[0] += u[t][e];
            }
            if (mine && c0 + t * TPR < nchunk) store_stream<TS>((TS*)a.y + at + c, u[t]);
        }
        if (a.pre) {
            float mean = 0.f;
            if (a.pre == CHIMERA_NORM_LAYER) {
                row_sums<TPR>(s, lds[odd][2], wave, lane);
                mean = s[0] * inv_cols;
            }
            s[0] = 0.f;
#pragma unroll
            for (int t = 0; t < MAXT; ++t)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    u[t][e] -= mean;
                    if (c0 + t * TPR < nchunk) s[0] += u[t][e] * u[t][e];
                }
            row_sums<TPR>(s, lds[odd][3], wave, lane);
            const float rstd = 1.0f / sqrtf(s[0] * inv_cols + a.eps);
            if (mine && c0 == 0) { a.stats[2 * (size_t)a.rows + row] = mean; a.stats[3 * (size_t)a.rows + row] = rstd; }
#pragma unroll
            for (int t = 0; t < MAXT; ++t) {
                const int c = min(c0 + t * TPR, nchunk - 1) * V;
                float g[V], b[V];
                load_elems<T, V>((const T*)a.pre_gain + c, g);
                if (a.pre_bias) load_elems<T, V>((const T*)a.pre_bias + c, b);
#pragma unroll
                for (int e = 0; e < V; ++e) u[t][e] = u[t][e] * rstd * g[e] + (a.pre_bias ? b[e] : 0.f);
                if (mine && c0 + t * TPR < nchunk) store_elems<T, V>((T*)a.h + at + c, u[t]);
            }
        }
    }
}

// --------------------------------------------------------------------- backward
// A workgroup takes `per_group` rows, as many side by side as it has threads for.  A thread's columns are the same in every row, so its share of the column sums
// stays in registers; at the end the rows side by side meet in LDS, in their order, and the workgroup's sums leave for join_sum_kernel (or are final
// where there is one workgroup).  dgate's sums end where a run of the gate ends: either a run holds whole workgroups, or a workgroup holds whole runs, and then
// each of the rows side by side belongs to a run of its own.
// A row is a chain of loads and two sums over its threads: the next row is asked for before the sums of this one, and small workgroups, two on a CU, fill one another's
// waits (8192 x 1600 bf16, all sums: 512 workgroups of 256 threads 50 us, 256 of 512 54; two rows at a time in each take the registers of the second
// workgroup, 71).
constexpr int bwd_threads(int threads_a_row) { return threads_a_row > 256 ? threads_a_row : 256; }
template <typename T, typename TS, int TPR, int MAXT>
__global__ __launch_bounds__(bwd_threads(TPR)) void join_bwd_kernel(JoinArgs a) {
    constexpr int LANES = bwd_threads(TPR) / TPR;           // rows side by side
    __shared__ float lds[2][2][2 * 8];
    extern __shared__ float meet_at[];                      // [LANES][cols], where LANES > 1
    const int tid = threadIdx.x, lane = tid % WAVE, wave = tid / WAVE, c0 = tid % TPR, rl = tid / TPR, cols = a.cols, nchunk = cols / V;
    const float inv_cols = 1.0f / (float)cols;
    // rows of the workgroup: whole runs of the gate, or a part of one
    int first, last;
    if (a.whole_runs || !a.gate) {
        first = blockIdx.x * a.per_group;
        last = min(a.rows, first + a.per_group);
    } else {
        const int run = blockIdx.x / a.groups_per_run;
        first = run * a.run + blockIdx.x % a.groups_per_run * a.per_group;
        last = min((run + 1) * a.run, first + a.per_group);
    }
    // of those, a lane takes every LANES-th, or (whole runs) neighbouring ones that are whole runs too
    const int own = a.whole_runs ? ((last - first) / a.run + LANES - 1) / LANES * a.run : 0;
    const int steps = a.whole_runs ? own : (last - first + LANES - 1) / LANES;
    auto row_of = [&](int i) { return a.whole_runs ? first + rl * own + i : first + i * LANES + rl; };
    int at[MAXT];                                           // the thread's columns; beyond the last ones: none
    bool live[MAXT];
    float gain1[MAXT][V], bias1[MAXT][V], gain2[MAXT][V], gate[MAXT][V];
#pragma unroll
    for (int t = 0; t < MAXT; ++t) {
        live[t] = c0 + t * TPR < nchunk;
        at[t] = live[t] ? (c0 + t * TPR) * V : 0;
#pragma unroll
        for (int e = 0; e < V; ++e) { gain1[t][e] = 1.f; bias1[t][e] = 0.f; gain2[t][e] = 0.f; gate[t][e] = 1.f; }
    }
    auto parameters = [&] {
#pragma unroll
        for (int t = 0; t < MAXT; ++t) {
            if (a.post) load_elems<T, V>((const T*)a.post_gain + at[t], gain1[t]);
            if (a.post_bias) load_elems<T, V>((const T*)a.post_bias + at[t], bias1[t]);
            if (a.pre) load_elems<T, V>((const T*)a.pre_gain + at[t], gain2[t]);
            if (a.gate && !a.whole_runs) load_elems<T, V>((const T*)a.gate + (size_t)(first / a.run) * cols + at[t], gate[t]);
        }
    };
    if constexpr (MAXT == 1) parameters();                  // (two chunks have no registers for them from row to row)
    float sum[SUMS][MAXT][V];
#pragma unroll
    for (int k = 0; k < SUMS; ++k)
#pragma unroll
        for (int t = 0; t < MAXT; ++t)
#pragma unroll
            for (int e = 0; e < V; ++e) sum[k][t][e] = 0.f;
    Chunk<T> rf[MAXT], rdh[MAXT], rg[MAXT];
    Chunk<TS> ry[MAXT], rdy[MAXT];
    float mean1 = 0.f, rstd1 = 1.f, mean2 = 0.f, rstd2 = 0.f;
    auto load = [&](int i) {
        const int row = min(row_of(i), last - 1);
#pragma unroll
        for (int t = 0; t < MAXT; ++t) {
            const size_t c = (size_t)row * cols + at[t];
            if (a.dy) rdy[t].load((const TS*)a.dy + c);
            if (a.pre) {
                rdh[t].load((const T*)a.dh + c);
                ry[t].load((const TS*)a.y + c);
            }
            rf[t].load((const T*)a.f + c);
            if (a.whole_runs) rg[t].load((const T*)a.gate + (size_t)(row / a.run) * cols + at[t]);
        }
        if (a.pre == CHIMERA_NORM_LAYER) mean2 = a.stats[2 * (size_t)a.rows + row];
        if (a.pre) rstd2 = a.stats[3 * (size_t)a.rows + row];
        if (a.post == CHIMERA_NORM_LAYER) mean1 = a.stats[row];
        if (a.post) rstd1 = a.stats[(size_t)a.rows + row];
    };
    load(0);
    for (int i = 0; i < steps; ++i) {
        const int row = row_of(i);
        const bool mine = row < last;                       // the same for the threads of a row
        const float m1 = mean1, r1 = rstd1, m2 = mean2, r2 = rstd2;
        float d[MAXT][V], hat1[MAXT][V], hat2[MAXT][V], dg[MAXT][V];
        if constexpr (MAXT > 1) parameters();
#pragma unroll
        for (int t = 0; t < MAXT; ++t) {
#pragma unroll
            for (int e = 0; e < V; ++e) { d[t][e] = 0.f; hat2[t][e] = 0.f; dg[t][e] = 0.f; }
            if (a.dy) rdy[t].unpack(d[t]);
            if (a.pre) {
                rdh[t].unpack(dg[t]);
                ry[t].unpack(hat2[t]);
            }
            rf[t].unpack(hat1[t]);
            if (a.whole_runs) rg[t].unpack(gate[t]);
        }
        if (i + 1 < steps) load(i + 1);
        if (a.pre) {
            float s[2] = {0.f, 0.f};
#pragma unroll
            for (int t = 0; t < MAXT; ++t)
                if (mine && live[t])
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        hat2[t][e] = (hat2[t][e] - m2) * r2;
                        sum[SUM_GAIN2][t][e] += dg[t][e] * hat2[t][e];
                        sum[SUM_BIAS2][t][e] += dg[t][e];
                        dg[t][e] *= gain2[t][e];
                        s[0] += dg[t][e];
                        s[1] += dg[t][e] * hat2[t][e];
                    }
            row_sums<TPR>(s, lds[i & 1][0], wave, lane);
            const float mean_d = a.pre == CHIMERA_NORM_LAYER ? s[0] * inv_cols : 0.f, c1 = s[1] * inv_cols;
#pragma unroll
            for (int t = 0; t < MAXT; ++t)
#pragma unroll
                for (int e = 0; e < V; ++e) d[t][e] += r2 * (dg[t][e] - mean_d - hat2[t][e] * c1);
        }
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int t = 0; t < MAXT; ++t)
            if (mine && live[t]) {
                if (a.dx) {
                    float o[V];
#pragma unroll
                    for (int e = 0; e < V; ++e) o[e] = a.alpha * d[t][e];
                    store_stream<TS>((TS*)a.dx + (size_t)row * cols + at[t], o);
                }
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    hat1[t][e] = (hat1[t][e] - m1) * r1;    // (without a norm: f itself)
                    d[t][e] *= a.beta;
                    sum[SUM_GATE][t][e] += d[t][e] * (hat1[t][e] * gain1[t][e] + bias1[t][e]);
                    d[t][e] *= gate[t][e];
                    sum[SUM_GAIN1][t][e] += d[t][e] * hat1[t][e];
                    sum[SUM_BIAS1][t][e] += d[t][e];
                    d[t][e] *= gain1[t][e];
                    s[0] += d[t][e];
                    s[1] += d[t][e] * hat1[t][e];
                }
            }
        if (a.whole_runs && (i + 1) % a.run == 0)                       // the end of a run: its row of dgate is this lane's
#pragma unroll
            for (int t = 0; t < MAXT; ++t) {
                if (mine && live[t] && a.out[SUM_GATE]) {
                    float* o = a.out[SUM_GATE] + (size_t)(row / a.run) * cols + at[t];
                    float v[V];
                    if (!a.overwrite) load_elems<float, V>(o, v);
#pragma unroll
                    for (int e = 0; e < V; ++e) v[e] = a.overwrite ? sum[SUM_GATE][t][e] : v[e] + sum[SUM_GATE][t][e];
                    store_elems<float, V>(o, v);
                }
#pragma unroll
                for (int e = 0; e < V; ++e) sum[SUM_GATE][t][e] = 0.f;
            }
        if (a.post) {
            row_sums<TPR>(s, lds[i & 1][1], wave, lane);
            const float mean_d = a.post == CHIMERA_NORM_LAYER ? s[0] * inv_cols : 0.f, c1 = s[1] * inv_cols;
#pragma unroll
            for (int t = 0; t < MAXT; ++t)
#pragma unroll
                for (int e = 0; e < V; ++e) d[t][e] = r1 * (d[t][e] - mean_d - hat1[t][e] * c1);
        }
        if (mine)
#pragma unroll
            for (int t = 0; t < MAXT; ++t)
                if (live[t]) store_elems<T, V>((T*)a.df + (size_t)row * cols + at[t], d[t]);
    }
    int slot = 0;
#pragma unroll
    for (int k = 0; k < SUMS; ++k) {
        if (!(a.sums >> k & 1)) continue;                               // the same for every thread
        if constexpr (LANES > 1) {
            __syncthreads();
#pragma unroll
            for (int t = 0; t < MAXT; ++t)
                if (live[t]) store_elems<float, V>(meet_at + (size_t)rl * cols + at[t], sum[k][t]);
            __syncthreads();
        }
        if (rl == 0)
#pragma unroll
            for (int t = 0; t < MAXT; ++t) {
                if (!live[t]) continue;
                float v[V];
#pragma unroll
                for (int e = 0; e < V; ++e) v[e] = sum[k][t][e];
                for (int l = 1; l < LANES; ++l) {
                    float w[V];
                    load_elems<float, V>(meet_at + (size_t)l * cols + at[t], w);
#pragma unroll
                    for (int e = 0; e < V; ++e) v[e] += w[e];
                }
                float* o = a.partial ? a.partial + ((size_t)blockIdx.x * __builtin_popcount(a.sums) + slot) * cols + at[t] : a.out[k] + at[t];
                if (!a.partial && !a.overwrite) {
                    float w[V];
                    load_elems<float, V>(o, w);
#pragma unroll
                    for (int e = 0; e < V; ++e) v[e] += w[e];
                }
                store_elems<float, V>(o, v);
            }
        ++slot;
    }
}

// The workgroups' sums, in their order: 32 sub-sums of every 32nd workgroup, then those.  blockIdx.y: which sum; from `slots` on, rows of dgate, whose
// workgroups lie together.
struct JoinSums {
    const float* partial;
    float* out[SUMS];                    // of the slots
    int slots, cols, groups, gate_slot, groups_per_run, overwrite;
};
__global__ __launch_bounds__(1024) void join_sum_kernel(JoinSums a) {
    __shared__ float red[32][32];
    const int c = threadIdx.x & 31, q = threadIdx.x >> 5, i = blockIdx.x * 32 + c, y = blockIdx.y;
    const bool gate = a.gate_slot >= 0 && y >= a.gate_slot;             // the gate's sum is the last slot
    const int run = gate ? y - a.gate_slot : 0, first = gate ? run * a.groups_per_run : 0, count = gate ? a.groups_per_run : a.groups;
    const int slot = gate ? a.gate_slot : y;
    const float* p = a.partial + ((size_t)first * a.slots + slot) * a.cols + i;
    const size_t step = (size_t)a.slots * a.cols;
    float s = 0.f;
    if (i < a.cols) {
        int g = q;
        for (; g + 96 < count; g += 128) s += (p[g * step] + p[(g + 32) * step]) + (p[(g + 64) * step] + p[(g + 96) * step]);
        for (; g < count; g += 32) s += p[g * step];
    }
    red[q][c] = s;
    __syncthreads();
    if (q == 0 && i < a.cols) {
        float t = red[0][c];
#pragma unroll
        for (int k = 1; k < 32; ++k) t += red[k][c];
        float* o = a.out[slot] + (size_t)run * a.cols + i;
        *o = a.overwrite ? t : *o + t;
    }
}

// ------------------------------------------------------------------------- host
#define JOIN_TRY(expr) do { int rc__ = (expr); if (rc__) return rc__; } while (0)

int threads_a_row(int cols) { return cols <= 512 ? 64 : cols <= 1024 ? 128 : cols <= 2048 ? 256 : 512; }

// Rows of a workgroup, workgroups, and how runs of the gate and workgroups hold one another
struct BwdPlan { int per_group, groups, whole_runs, groups_per_run; };
BwdPlan bwd_plan(int rows, int cols, int gate_rows) {
    BwdPlan p{};
    const int lanes = bwd_threads(threads_a_row(cols)) / threads_a_row(cols);
    // no more than 8 rows a lane: one workgroup, whose sums are final (a launch less)
    const int per = rows <= 8 * lanes ? rows : (std::max((rows + ROW_GROUPS - 1) / ROW_GROUPS, lanes) + lanes - 1) / lanes * lanes;
    if (!gate_rows) {
        p.per_group = per;
        p.groups = (rows + per - 1) / per;
        return p;
    }
    const int run = rows / gate_rows;
    if (run >= per) {
        p.groups_per_run = (run + per - 1) / per;
        p.per_group = (run + p.groups_per_run - 1) / p.groups_per_run;
        p.groups = p.groups_per_run * gate_rows;
        return p;
    }
    p.whole_runs = 1;
    p.per_group = std::max(per / run, 1) * run;
    p.groups = (rows + p.per_group - 1) / p.per_group;
    return p;
}
size_t bwd_bytes(int rows, int cols, int gate_rows) { return (size_t)bwd_plan(rows, cols, gate_rows).groups * SUMS * cols * 4; }

int check_join(int dtype, int stream_dtype, int rows, int cols, int gate_rows, int post, int pre) {
    if (dtype != CHIMERA_F32 && dtype != CHIMERA_BF16) return fail(CHIMERA_EINVAL, "unknown dtype %d", dtype);
    if (stream_dtype != CHIMERA_F32 && stream_dtype != dtype) return fail(CHIMERA_EINVAL, "the stream is float or of the branch's type");
    if (rows < 1 || cols < 1) return fail(CHIMERA_EINVAL, "sizes must be positive");
    if (cols % 8 || cols > BN_COLS) return fail(CHIMERA_EINVAL, "cols=%d must be a multiple of 8 up to %d", cols, BN_COLS);
    if (rows > 1 << 28) return fail(CHIMERA_EINVAL, "more than 2^28 rows");
    if (gate_rows < 0 || (gate_rows && rows % gate_rows)) return fail(CHIMERA_EINVAL, "gate_rows=%d must divide rows=%d", gate_rows, rows);
    if (post < CHIMERA_NORM_NONE || post > CHIMERA_NORM_RMS || pre < CHIMERA_NORM_NONE || pre > CHIMERA_NORM_RMS) return fail(CHIMERA_EINVAL, "unknown norm");
    return CHIMERA_OK;
}

#define JOIN_SIZES(GO, T, TS)                                                                                 \
    do {                                                                                                      \
        if (cols <= 512) GO(T, TS, 64, 1);                                                                    \
        else if (cols <= 1024) GO(T, TS, 128, 1);                                                             \
        else if (cols <= 2048) GO(T, TS, 256, 1);                                                             \
        else if (cols <= 4096) GO(T, TS, WIDE, 4096 / 8 / WIDE);                                              \
        else GO(T, TS, WIDE, 8192 / 8 / WIDE);                                                                \
    } while (0)
#define JOIN_TYPES(GO)                                                                                        \
    do {                                                                                                      \
        if (dtype == CHIMERA_F32) JOIN_SIZES(GO, float, float);                                               \
        else if (stream_dtype == CHIMERA_F32) JOIN_SIZES(GO, bf16_t, float);                                  \
        else JOIN_SIZES(GO, bf16_t, bf16_t);                                                                  \
    } while (0)

}  // namespace

}  // namespace chimera

using namespace chimera;

extern "C" {

int chimera_op_branch_norm_fwd(int dtype, int stream_dtype, int rows, int cols, int post, int pre, float eps, float alpha, float beta, const void* d_f,
                               const void* d_x, const void* d_gate, int gate_rows, const void* d_post_gain, const void* d_post_bias, const void* d_pre_gain,
                               const void* d_pre_bias, void* d_y, void* d_h, float* d_stats, void* hip_stream) {
    if (!d_gate) gate_rows = 0;
    JOIN_TRY(check_join(dtype, stream_dtype, rows, cols, gate_rows, post, pre));
    if (d_gate && !gate_rows) return fail(CHIMERA_EINVAL, "a gate of no rows");
    if (!(eps >= 0) || !std::isfinite(eps) || !std::isfinite(alpha) || !std::isfinite(beta)) return fail(CHIMERA_EINVAL, "eps, alpha and beta must be finite, eps not negative");
    if (!d_f || !d_y || (post && !d_post_gain) || (pre && (!d_pre_gain || !d_h)) || ((post || pre) && !d_stats)) return fail(CHIMERA_EINVAL, "NULL operand");
    if (!post) d_post_gain = d_post_bias = nullptr;
    if (!pre) d_pre_gain = d_pre_bias = nullptr, d_h = nullptr;
    if (((uintptr_t)d_f | (uintptr_t)d_x | (uintptr_t)d_gate | (uintptr_t)d_post_gain | (uintptr_t)d_post_bias | (uintptr_t)d_pre_gain | (uintptr_t)d_pre_bias |
         (uintptr_t)d_y | (uintptr_t)d_h) & 15 || (uintptr_t)d_stats & 3) return fail(CHIMERA_EINVAL, "tensors must be 16-byte aligned");
    const size_t e = dtype == CHIMERA_F32 ? 4 : 2, es = stream_dtype == CHIMERA_F32 ? 4 : 2, n = (size_t)rows * cols, c = (size_t)cols * e;
    const Rows y = plain(d_y, n * es), h = plain(d_h, n * e), stats = plain(post || pre ? d_stats : nullptr, (size_t)rows * 16);
    JOIN_TRY(check_apart({plain(d_gate, (size_t)gate_rows * c), plain(d_post_gain, c), plain(d_post_bias, c), plain(d_pre_gain, c), plain(d_pre_bias, c)}, {y, h, stats}));
    // (a row is written when it has been read: y may take the place of x, and h that of f)
    JOIN_TRY(check_apart({plain(d_x, n * es)}, {d_y == d_x ? plain(nullptr, 1) : y, h, stats}));
    JOIN_TRY(check_apart({plain(d_f, n * e)}, {y, d_h == d_f ? plain(nullptr, 1) : h, stats}));
    JoinArgs a{};
    a.rows = rows; a.cols = cols; a.run = gate_rows ? rows / gate_rows : 1; a.post = post; a.pre = pre; a.eps = eps; a.alpha = alpha; a.beta = beta;
    a.f = d_f; a.x = d_x; a.gate = d_gate; a.post_gain = d_post_gain; a.post_bias = d_post_bias; a.pre_gain = d_pre_gain; a.pre_bias = d_pre_bias;
    a.y = d_y; a.h = d_h; a.stats = d_stats;
    constexpr int WIDE = 256;
    const int lanes = 256 / std::min(threads_a_row(cols), 256);
    a.per_group = std::max(lanes, (rows + 8191) / 8192 * lanes);
    const dim3 grid((unsigned)((rows + a.per_group - 1) / a.per_group));
    hipStream_t s = (hipStream_t)hip_stream;
#define JOIN_FWD(T, TS, TPR, MAXT) hipLaunchKernelGGL((join_fwd_kernel<T, TS, TPR, MAXT>), grid, dim3(256), 0, s, a)
    JOIN_TYPES(JOIN_FWD);
    CHIMERA_LAUNCH_CHECK("norm of a branch");
    return CHIMERA_OK;
}

size_t chimera_op_branch_norm_bwd_workspace_bytes(int rows, int cols, int gate_rows) {
    return check_join(CHIMERA_F32, CHIMERA_F32, rows, cols, gate_rows, 0, 0) ? 0 : bwd_bytes(rows, cols, gate_rows);
}

int chimera_op_branch_norm_bwd(int dtype, int stream_dtype, int rows, int cols, int post, int pre, float alpha, float beta, const void* d_f, const void* d_y,
                               const void* d_gate, int gate_rows, const void* d_post_gain, const void* d_post_bias, const void* d_pre_gain, const float* d_stats,
                               const void* d_dy, const void* d_dh, void* d_dx, void* d_df, float* d_dpost_gain, float* d_dpost_bias, float* d_dpre_gain,
                               float* d_dpre_bias, float* d_dgate, int overwrite, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
    if (!d_gate) gate_rows = 0;
    JOIN_TRY(check_join(dtype, stream_dtype, rows, cols, gate_rows, post, pre));
    if (d_gate && !gate_rows) return fail(CHIMERA_EINVAL, "a gate of no rows");
    if (!std::isfinite(alpha) || !std::isfinite(beta)) return fail(CHIMERA_EINVAL, "alpha and beta must be finite");
    if (!d_f || !d_df || !d_workspace || (post && !d_post_gain) || (pre && (!d_pre_gain || !d_y || !d_dh)) || ((post || pre) && !d_stats)) return fail(CHIMERA_EINVAL, "NULL operand");
    if (!pre && !d_dy) return fail(CHIMERA_EINVAL, "no gradient comes in");
    if ((!post && (d_dpost_gain || d_dpost_bias)) || (!pre && (d_dpre_gain || d_dpre_bias)) || (!d_gate && d_dgate))
        return fail(CHIMERA_EINVAL, "a gradient of what the call does not have");
    if (!post) d_post_gain = d_post_bias = nullptr;
    if (!pre) d_pre_gain = d_y = d_dh = nullptr;
    if (((uintptr_t)d_f | (uintptr_t)d_y | (uintptr_t)d_gate | (uintptr_t)d_post_gain | (uintptr_t)d_post_bias | (uintptr_t)d_pre_gain | (uintptr_t)d_dy | (uintptr_t)d_dh |
         (uintptr_t)d_dx | (uintptr_t)d_df | (uintptr_t)d_dpost_gain | (uintptr_t)d_dpost_bias | (uintptr_t)d_dpre_gain | (uintptr_t)d_dpre_bias | (uintptr_t)d_dgate) & 15 ||
        (uintptr_t)d_stats & 3 || (uintptr_t)d_workspace & 255) return fail(CHIMERA_EINVAL, "tensors must be 16-byte aligned, the workspace 256-byte aligned");
    const size_t need = bwd_bytes(rows, cols, gate_rows);
    if (workspace_bytes < need) return fail(CHIMERA_ENOMEM, "workspace holds %zu bytes, need %zu", workspace_bytes, need);
    const size_t e = dtype == CHIMERA_F32 ? 4 : 2, es = stream_dtype == CHIMERA_F32 ? 4 : 2, n = (size_t)rows * cols, c = (size_t)cols * e, c4 = (size_t)cols * 4;
    const Rows dx = plain(d_dx, n * es), df = plain(d_df, n * e), g1 = plain(d_dpost_gain, c4), b1 = plain(d_dpost_bias, c4), g2 = plain(d_dpre_gain, c4),
               b2 = plain(d_dpre_bias, c4), dgate = plain(d_dgate, gate_rows * c4), ws = plain(d_workspace, need), none = plain(nullptr, 1);
    JOIN_TRY(check_apart({plain(d_f, n * e), plain(d_y, n * es), plain(d_gate, gate_rows * c), plain(d_post_gain, c), plain(d_post_bias, c), plain(d_pre_gain, c),
                          plain(post || pre ? d_stats : nullptr, (size_t)rows * 16)}, {dx, df, g1, b1, g2, b2, dgate, ws}));
    // (a row is written when it has been read: dx may take the place of dy, and df that of dh)
    JOIN_TRY(check_apart({plain(d_dy, n * es)}, {d_dx == d_dy ? none : dx, df, g1, b1, g2, b2, dgate, ws}));
    JOIN_TRY(check_apart({plain(d_dh, n * e)}, {dx, d_df == d_dh ? none : df, g1, b1, g2, b2, dgate, ws}));
    JoinArgs a{};
    a.rows = rows; a.cols = cols; a.run = gate_rows ? rows / gate_rows : 1; a.post = post; a.pre = pre; a.alpha = alpha; a.beta = beta;
    a.f = d_f; a.gate = d_gate; a.post_gain = d_post_gain; a.post_bias = d_post_bias; a.pre_gain = d_pre_gain; a.y = (void*)d_y; a.stats = (float*)d_stats;
    a.dy = d_dy; a.dh = d_dh; a.dx = d_dx; a.df = d_df; a.overwrite = overwrite;
    const BwdPlan p = bwd_plan(rows, cols, gate_rows);
    a.per_group = p.per_group; a.whole_runs = p.whole_runs; a.groups_per_run = p.groups_per_run;
    float* outs[SUMS] = {d_dpost_gain, d_dpost_bias, d_dpre_gain, d_dpre_bias, d_dgate};
    JoinSums r{};
    r.gate_slot = -1;
    for (int k = 0; k < SUMS; ++k) {
        a.out[k] = outs[k];
        if (!outs[k] || (k == SUM_GATE && p.whole_runs)) continue;
        a.sums |= 1 << k;
        if (k == SUM_GATE) r.gate_slot = r.slots;
        r.out[r.slots++] = outs[k];
    }
    a.partial = p.groups > 1 ? (float*)d_workspace : nullptr;
    constexpr int WIDE = 512;
    const int lanes = bwd_threads(threads_a_row(cols)) / threads_a_row(cols);
    const size_t lds = lanes > 1 ? (size_t)lanes * cols * 4 : 0;
    hipStream_t s = (hipStream_t)hip_stream;
#define JOIN_BWD(T, TS, TPR, MAXT) hipLaunchKernelGGL((join_bwd_kernel<T, TS, TPR, MAXT>), dim3((unsigned)p.groups), dim3(bwd_threads(TPR)), lds, s, a)
    JOIN_TYPES(JOIN_BWD);
    CHIMERA_LAUNCH_CHECK("norm of a branch, backward");
    if (a.partial && r.slots) {
        r.partial = a.partial; r.cols = cols; r.groups = p.groups; r.groups_per_run = p.groups_per_run; r.overwrite = overwrite;
        const unsigned ny = (unsigned)(r.gate_slot >= 0 ? r.gate_slot + gate_rows : r.slots);
        hipLaunchKernelGGL(join_sum_kernel, dim3((unsigned)((cols + 31) / 32), ny), dim3(1024), 0, s, r);
        CHIMERA_LAUNCH_CHECK("norm of a branch, backward");
    }
    return CHIMERA_OK;
}

}  // extern "C"
