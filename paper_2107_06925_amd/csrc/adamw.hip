// The step from gradients to weights, over many tensors at once: the norm of all gradients with the factor that clips them, and
// AdamW with moments in 32 or in 8 bits.
//   g' = factor g,  m = b1 m + (1 - b1) g',  v = b2 v + (1 - b2) g'^2,  r = sqrt(v)
//   p = p (1 - lr decay) - lr / (1 - b1^t) m / (r / sqrt(1 - b2^t) + eps)
// What bounds both is memory: a value's 28 bytes (float), 30 (bf16 with a float master weight) or 18 (the same with 8-bit moments), and 4 for the norm.
// The tensors' addresses travel as a kernel argument, so a launch takes some tens of them and nothing has to be laid out in device memory.
//
// 8-bit moments: m and r are held as e4m3 numbers times a float scale for each 256 values, the largest of which becomes 448.  r and not v: its
// range is the root of v's, and a code's range of 2^17.8 then spans one of 2^35 in v.  Codes are rounded at random (up with the probability that
// keeps the expectation): a step moves r by less than a thousandth, a code is 6 to 12 % wide, and rounding to nearest would leave r where it is for good.
// The random bits are a hash of (seed, step, the value's number), so a step's result is a function of its arguments.  A value whose r is
// not zero keeps a code above zero, whatever the bits: its m would otherwise be divided by eps.
#include "device.h"

#include <algorithm>
#include <cfloat>
#include <climits>
#include <cmath>
#include <new>

namespace chimera {
namespace {

constexpr int STEP_THREADS = 256, MOMENT_BLOCK = 256;
static_assert(MOMENT_BLOCK == 4 * WAVE, "a wavefront holds one block of moments, four values a lane");
constexpr float CODE_TOP = 448.0f, CODE_LEAST = 1e-30f;      // largest e4m3 number; blocks whose largest value is below this hold zeros

// Tensors need not be aligned to more than their elements.
typedef float f4_t __attribute__((ext_vector_type(4)));
typedef f4_t f4_u __attribute__((aligned(4)));
typedef bf16_t b4_t __attribute__((ext_vector_type(4)));
typedef b4_t b4_u __attribute__((aligned(2)));
typedef unsigned u32_u __attribute__((aligned(1)));

struct Scalars { float b1, w1, b2, w2, eps, lr, rate, root; unsigned key; };     // w = 1 - b, rate = lr / (1 - b1^t), root = 1 / sqrt(1 - b2^t)
__host__ __device__ Scalars scalars_of(const chimera_adamw_hyper& h) {
    Scalars s;
    s.b1 = (float)h.beta1; s.w1 = (float)(1.0 - h.beta1); s.b2 = (float)h.beta2; s.w2 = (float)(1.0 - h.beta2);
    s.eps = (float)h.eps; s.lr = (float)h.lr;
    s.rate = (float)(h.lr / (1.0 - pow(h.beta1, (double)h.step)));
    s.root = (float)(1.0 / sqrt(1.0 - pow(h.beta2, (double)h.step)));
    // all 64 bits of both.  (Odd numbers from pi and e, and from the roots of 11 and 17; below from the golden ratio and the roots of 2 and 3.)
    s.key = (unsigned)h.seed * 0x243F6A89u + (unsigned)h.step * 0xB7E15163u + (unsigned)(h.seed >> 32) * 0x510E527Fu + (unsigned)((uint64_t)h.step >> 32) * 0x1F83D9ABu;
    return s;
}
struct DeviceHyper { chimera_adamw_hyper given; Scalars derived; };
static_assert(sizeof(DeviceHyper) <= CHIMERA_ADAMW_HYPER_BYTES, "room for what a call derives");
__global__ void adamw_derive_kernel(DeviceHyper* h) { h->derived = scalars_of(h->given); }

constexpr int STEP_TENSORS = 48;
struct StepTensor {
    void *p, *m, *v;
    float *master, *scale;
    const float* g;
    long long n;
    long long block0;            // number of the tensor's first block of 256 values in the call
    float decay;
};
struct StepLaunch {
    StepTensor t[STEP_TENSORS];
    int first[STEP_TENSORS];     // a tensor's first chunk (INT_MAX behind the last tensor)
    Scalars s;
    int chunk;                   // values per workgroup
    const DeviceHyper* device;   // null: s
    const float* factor;
};
static_assert(sizeof(StepLaunch) <= 4096, "kernel arguments");

// Number of the last tensor that begins at or before `chunk` (lanes ask for 64 beginnings at once).
template <int N> __device__ __forceinline__ int tensor_of(const int (&first)[N], int chunk) {
    static_assert(N <= WAVE, "one lane a tensor");
    const int lane = threadIdx.x % WAVE;
    const bool at = lane < N && first[min(lane, N - 1)] <= chunk;
    return __builtin_amdgcn_readfirstlane(__popcll(__ballot(at)) - 1);
}

// of value i: mixed(start(i, key)), and i + 1 starts RANDOM_STEP later
constexpr unsigned RANDOM_STEP = 0x9E3779B1u;
__device__ __forceinline__ unsigned random_start(unsigned long long i, unsigned key) { return (unsigned)i * RANDOM_STEP + (unsigned)(i >> 32) * 0x6A09E667u + key; }
__device__ __forceinline__ unsigned mixed(unsigned x) {
    x = (x ^ (x >> 15)) * 0x6A09E667u;
    x = (x ^ (x >> 13)) * 0xBB67AE85u;
    return x ^ (x >> 16);
}
// |x| / top as an e4m3 code: its bits follow from the float's, whose exponent is moved so that e4m3's smallest normal number becomes the float's.
__device__ __forceinline__ unsigned encode(float x, float inv, unsigned bits16, bool keep) {
#pragma clang fp contract(off)
    const float y = fabsf(x) * inv;
    if (!(y <= FLT_MAX)) return 0x7f;                         // not a number stays one, and e4m3 has no infinities
    unsigned code = min((__float_as_uint(y * 0x1p-120f) + bits16 * 16u + 8u) >> 20, 126u);
    if (keep && x > 0.f) code = max(code, 1u);
    return x < 0.f ? code | 0x80u : code;
}
__device__ __forceinline__ float decode(unsigned code, float scale) {
    const float v = __uint_as_float((code & 0x7f) << 20) * 0x1p120f;
    return ((code & 0x7f) == 0x7f ? __builtin_nanf("") : code & 0x80 ? -v : v) * scale;
}

// Every operation on the moments is rounded by itself (no contraction), so that the choice of codes is a function of the numbers; the update's quotient takes the
// hardware's reciprocal (1 ulp), half of a correctly rounded division's instructions: they are what the 8-bit step is short of beside memory.
// ONCE: what a step touches is more than the memory-side cache holds, and passes it by.
// 184 million bf16 weights 969 us, 5.7 TB/s (a large copy 5.2); 101 million with 8-bit moments 330 us, 5.5 TB/s; 397 thousand float ones 4.6 us, a launch and one trip.
template <typename T, int BITS, bool ONCE>
__global__ __launch_bounds__(STEP_THREADS) void adamw_kernel(StepLaunch L) {
#pragma clang fp contract(off)
    const float factor = L.factor ? *L.factor : 1.0f;
    if (!(fabsf(factor) <= 3.4028235e38f)) return;            // not finite: nothing changes
    const Scalars s = L.device ? L.device->derived : L.s;
    const int k = tensor_of(L.first, (int)blockIdx.x);
    const StepTensor& t = L.t[k];
    const long long n = t.n, begin = (long long)((int)blockIdx.x - L.first[k]) * L.chunk, end = min(begin + L.chunk, n);
    const float keep = 1.0f - t.decay * s.lr;
    T* __restrict__ const param = (T*)t.p;
    float* __restrict__ const weight = sizeof(T) == 4 ? (float*)t.p : t.master;
    const float* __restrict__ const grad = t.g;
    const int lane = threadIdx.x % WAVE;
    for (long long i0 = begin + threadIdx.x / WAVE * MOMENT_BLOCK; i0 < end; i0 += STEP_THREADS / WAVE * MOMENT_BLOCK) {
        const long long i = i0 + lane * 4;
        const int have = (int)max(0ll, min(4ll, n - i));     // of this lane's four values
        f4_t g = {0.f, 0.f, 0.f, 0.f}, w = g, m = g, v = g, r;
        auto get = [&](const float* from, f4_t& to) {
            if (have == 4) {
                if constexpr (ONCE) to = __builtin_nontemporal_load(reinterpret_cast<const f4_u*>(from + i));
                else to = *reinterpret_cast<const f4_u*>(from + i);
            } else
#pragma unroll
                for (int e = 0; e < 3; ++e)
                    if (e < have) to[e] = from[i + e];
        };
        auto put = [&](float* to, const f4_t& x) {
            if (have == 4) {
                if constexpr (ONCE) __builtin_nontemporal_store(x, reinterpret_cast<f4_u*>(to + i));
                else *reinterpret_cast<f4_u*>(to + i) = x;
            } else
#pragma unroll
                for (int e = 0; e < 3; ++e)
                    if (e < have) to[i + e] = x[e];
        };
        auto get_codes = [&](const void* from) {
            const unsigned char* c = (const unsigned char*)from + i;
            unsigned q = 0;
            if (have == 4) q = *reinterpret_cast<const u32_u*>(c);
            else
#pragma unroll
                for (int e = 0; e < 3; ++e)
                    if (e < have) q |= (unsigned)c[e] << (8 * e);
            return q;
        };
        auto put_codes = [&](void* to, unsigned q) {
            unsigned char* c = (unsigned char*)to + i;
            if (have == 4) *reinterpret_cast<u32_u*>(c) = q;
            else
#pragma unroll
                for (int e = 0; e < 3; ++e)
                    if (e < have) c[e] = (unsigned char)(q >> (8 * e));
        };
        get(grad, g);
        get(weight, w);
        if constexpr (BITS == 32) {
            get((const float*)t.m, m);
            get((const float*)t.v, v);
        } else {
            const unsigned qm = get_codes(t.m), qv = get_codes(t.v);
            const float sm = t.scale[i0 / MOMENT_BLOCK * 2], sv = t.scale[i0 / MOMENT_BLOCK * 2 + 1];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                m[e] = decode(qm >> (8 * e) & 0xff, sm);
                const float root = decode(qv >> (8 * e) & 0xff, sv);
                v[e] = root * root;
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float x = g[e] * factor;
            m[e] = m[e] * s.b1 + x * s.w1;
            v[e] = v[e] * s.b2 + (x * x) * s.w2;
            r[e] = sqrtf(v[e]);                               // correctly rounded
            w[e] = w[e] * keep - (m[e] * s.rate) * __builtin_amdgcn_rcpf(r[e] * s.root + s.eps);
        }
        put(weight, w);
        if constexpr (sizeof(T) == 2) {
            if (have == 4) *reinterpret_cast<b4_u*>(param + i) = b4_t{(bf16_t)w[0], (bf16_t)w[1], (bf16_t)w[2], (bf16_t)w[3]};
            else
#pragma unroll
                for (int e = 0; e < 3; ++e)
                    if (e < have) param[i + e] = (bf16_t)w[e];
        }
        if constexpr (BITS == 32) {
            put((float*)t.m, m);
            put((float*)t.v, v);
        } else {
            float tm = 0.f, tv = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < have) { tm = fmaxf(tm, fabsf(m[e])); tv = fmaxf(tv, r[e]); }
            tm = wave_max(tm);
            tv = wave_max(tv);
            if (!(fmaxf(tm, tv) <= FLT_MAX)) {                // an infinite moment is not its block's scale, which would leave the others no value
                auto largest = [&](const f4_t& x) {
                    float top = 0.f;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (e < have && fabsf(x[e]) <= FLT_MAX) top = fmaxf(top, fabsf(x[e]));
                    return wave_max(top);
                };
                tm = largest(m);
                tv = largest(r);
            }
            const float im = tm > CODE_LEAST ? __fdiv_rn(1.0f, tm) * CODE_TOP : 0.f, iv = tv > CODE_LEAST ? __fdiv_rn(1.0f, tv) * CODE_TOP : 0.f;
            unsigned qm = 0, qv = 0;
            const unsigned start = random_start((unsigned long long)(t.block0 * MOMENT_BLOCK + i), s.key);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const unsigned bits = mixed(start + e * RANDOM_STEP);
                qm |= encode(m[e], im, bits & 0xffff, false) << (8 * e);
                qv |= encode(r[e], iv, bits >> 16, iv > 0.f) << (8 * e);
            }
            put_codes(t.m, qm);
            put_codes(t.v, qv);
            if (lane == 0) {
                t.scale[i0 / MOMENT_BLOCK * 2] = tm > CODE_LEAST ? tm * (1.0f / CODE_TOP) : 0.f;
                t.scale[i0 / MOMENT_BLOCK * 2 + 1] = tv > CODE_LEAST ? tv * (1.0f / CODE_TOP) : 0.f;
            }
        }
    }
}

// ---- sum of squares: a double per workgroup, in a fixed order; one workgroup adds them.  (Squares of floats reach beyond the floats' range.)
// Bound by memory: 369 million values 246 us, 6.0 TB/s; 793 thousand 3.6 + 1.8 us, a launch's latency each.
constexpr int NORM_TENSORS = 64;
struct NormLaunch {
    const float* g[NORM_TENSORS];
    long long n[NORM_TENSORS];
    int first[NORM_TENSORS];
    long long chunk;
    double* partial;
};
__device__ __forceinline__ double wave_sum_double(double v) {
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o, WAVE);
    return v;
}
__global__ __launch_bounds__(STEP_THREADS) void grad_square_kernel(NormLaunch L) {
    __shared__ double part[STEP_THREADS / WAVE];
    const int k = tensor_of(L.first, (int)blockIdx.x);
    const float* g = L.g[k];
    const long long begin = (long long)((int)blockIdx.x - L.first[k]) * L.chunk, end = min(begin + L.chunk, L.n[k]);
    double sum[4] = {0, 0, 0, 0};
    constexpr int FLY = 4, STRIDE = STEP_THREADS * 4;
    long long i = begin + threadIdx.x * 4;
    for (; i + (FLY - 1) * STRIDE + 4 <= end; i += FLY * STRIDE) {
        f4_t x[FLY];
#pragma unroll
        for (int u = 0; u < FLY; ++u) x[u] = *reinterpret_cast<const f4_u*>(g + i + u * STRIDE);
#pragma unroll
        for (int u = 0; u < FLY; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] += (double)x[u][e] * x[u][e];
    }
    for (; i < end; i += STRIDE)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (i + e < end) { const double x = g[i + e]; sum[e] += x * x; }
    const double s = wave_sum_double((sum[0] + sum[1]) + (sum[2] + sum[3]));
    if (threadIdx.x % WAVE == 0) part[threadIdx.x / WAVE] = s;
    __syncthreads();
    if (threadIdx.x == 0) L.partial[blockIdx.x] = (part[0] + part[1]) + (part[2] + part[3]);
}
__global__ __launch_bounds__(1024) void grad_norm_kernel(const double* __restrict__ partial, int n, float max_norm, float* __restrict__ out) {
    __shared__ double part[1024 / WAVE];
    double s = 0;
    for (int i = threadIdx.x; i < n; i += 1024) s += partial[i];
    s = wave_sum_double(s);
    if (threadIdx.x % WAVE == 0) part[threadIdx.x / WAVE] = s;
    __syncthreads();
    if (threadIdx.x) return;
    s = 0;
    for (int i = 0; i < 1024 / WAVE; ++i) s += part[i];
    const double norm = sqrt(s);
    out[0] = (float)norm;
    out[1] = !(norm <= 3.4028235e38) ? __builtin_nanf("") : norm > max_norm ? (float)(max_norm / norm) : 1.0f;
}

// Values per workgroup: eight workgroups a CU, pieces of at least 4096
constexpr long long NORM_CHUNKS = 2048;
bool norm_chunk(int count, const int64_t* h_n, long long& chunk) {
    long long total = 0;
    for (int i = 0; i < count; ++i) {
        if (h_n[i] < 0 || h_n[i] > 1ll << 40 || (total += h_n[i]) > 1ll << 40) return false;
    }
    chunk = std::max((total / NORM_CHUNKS + 1023) / 1024 * 1024, 4096ll);
    return true;
}
size_t norm_bytes(int count) { return ((size_t)NORM_CHUNKS + count) * sizeof(double); }

int check_hyper(const chimera_adamw_hyper& h) {
    if (!(h.lr >= 0) || !std::isfinite(h.lr)) return fail(CHIMERA_EINVAL, "lr must be finite and not negative");
    if (!(h.beta1 >= 0 && h.beta1 < 1) || !(h.beta2 >= 0 && h.beta2 < 1)) return fail(CHIMERA_EINVAL, "beta1 and beta2 must lie in [0, 1)");
    if (!(h.eps >= 0x1p-126) || !(h.eps <= 1)) return fail(CHIMERA_EINVAL, "eps must lie in [2^-126, 1]");
    if (h.step < 1) return fail(CHIMERA_EINVAL, "step=%lld: the first step is 1", (long long)h.step);
    return CHIMERA_OK;
}

// Spans of memory by kind, each kind `room` of them at most, the last only read: whether what is written shares a byte with anything else.  One walk over all in the
// order of addresses, of each kind, which usually lies sorted in a range of its own, as many as come before the next kind's.
struct Span {
    uintptr_t begin, end;
    bool operator<(const Span& o) const { return begin < o.begin; }
};
template <int KINDS> struct Spans {
    std::vector<Span> all;
    size_t room, count[KINDS] = {};
    explicit Spans(size_t room) : all(room * KINDS), room(room) {}
    void add(int kind, const void* p, size_t bytes) { if (p) all[kind * room + count[kind]++] = {(uintptr_t)p, (uintptr_t)p + bytes}; }
    bool written_twice() {
        struct Kind { Span *at, *end; bool read; } kinds[KINDS];
        int n = 0;
        for (int i = 0; i < KINDS; ++i) {
            Span *first = all.data() + i * room, *last = first + count[i];
            if (!std::is_sorted(first, last)) std::sort(first, last);
            if (first != last) kinds[n++] = {first, last, i == KINDS - 1};
        }
        uintptr_t written = 0, read = 0;                      // ends of what has been passed
        while (n) {
            int k = 0;
            for (int i = 1; i < n; ++i)
                if (*kinds[i].at < *kinds[k].at) k = i;
            Kind& next = kinds[k];
            uintptr_t others = UINTPTR_MAX;
            for (int i = 0; i < n; ++i)
                if (i != k) others = std::min(others, kinds[i].at->begin);
            do {
                if (next.at->begin < written || (!next.read && next.at->begin < read)) return true;
                uintptr_t& end = next.read ? read : written;
                end = std::max(end, next.at->end);
            } while (++next.at != next.end && next.at->begin <= others);
            if (next.at == next.end) next = kinds[--n];
        }
        return false;
    }
};

}  // namespace

int adamw_step(int dtype, int bits, int count, const AdamwTensor* t, const chimera_adamw_hyper* h_hyper, void* d_hyper, const float* d_factor, void* stream) {
    hipStream_t s = (hipStream_t)stream;
    StepLaunch L{};
    L.factor = d_factor;
    L.device = (const DeviceHyper*)d_hyper;
    if (d_hyper) {
        hipLaunchKernelGGL(adamw_derive_kernel, dim3(1), dim3(1), 0, s, (DeviceHyper*)d_hyper);
        CHIMERA_LAUNCH_CHECK("AdamW");
    } else {
        L.s = scalars_of(*h_hyper);
    }
    // 1024 values a workgroup, four a lane, and no loop: a workgroup that goes round takes a trip to memory each time.  8-bit steps go round twice, beyond 4
    // million values, where they are short of instructions.  Measured (184 million bf16 weights; 101 million with 8-bit moments), us: 4096 values 1062; 350,
    // 2048 1048; 343, 1024 1030; 356; past the caches 1045; 336, 1022; 335, 990; 346.  A float step of 400 000 values 6.4 -> 4.6.
    long long total = 0, block = 0;
    for (int i = 0; i < count; ++i) total += t[i].n;
    L.chunk = bits == 8 && total > 4 << 20 ? 2048 : 1024;
    const bool once = total * (bits == 8 ? 18 : 28) > 256ll << 20;
    auto chunks_of = [&](int i) { return (t[i].n + L.chunk - 1) / L.chunk; };
    for (int i = 0; i < count;) {
        std::fill(std::begin(L.first), std::end(L.first), INT_MAX);
        long long chunks = 0;
        int used = 0;
        for (; i < count && used < STEP_TENSORS && chunks + chunks_of(i) < 1 << 23; ++i) {
            if (!t[i].n) continue;
            L.t[used] = {t[i].p, t[i].m, t[i].v, t[i].master, t[i].scale, t[i].g, (long long)t[i].n, block, t[i].decay};
            L.first[used++] = (int)chunks;
            chunks += chunks_of(i);
            block += (t[i].n + MOMENT_BLOCK - 1) / MOMENT_BLOCK;
        }
        if (!used) continue;
        const dim3 grid((unsigned)chunks), threads(STEP_THREADS);
        auto launch = [&]<typename T, int BITS>() {
            if (once) hipLaunchKernelGGL((adamw_kernel<T, BITS, true>), grid, threads, 0, s, L);
            else hipLaunchKernelGGL((adamw_kernel<T, BITS, false>), grid, threads, 0, s, L);
        };
        if (dtype == CHIMERA_F32 && bits == 32) launch.template operator()<float, 32>();
        else if (dtype == CHIMERA_F32) launch.template operator()<float, 8>();
        else if (bits == 32) launch.template operator()<bf16_t, 32>();
        else launch.template operator()<bf16_t, 8>();
        CHIMERA_LAUNCH_CHECK("AdamW");
    }
    return CHIMERA_OK;
}

int adamw_check(int dtype, int bits, const chimera_adamw_hyper* h_hyper, const void* d_hyper) {
    if (dtype != CHIMERA_F32 && dtype != CHIMERA_BF16) return fail(CHIMERA_EINVAL, "unknown dtype %d", dtype);
    if (bits != 32 && bits != 8) return fail(CHIMERA_EINVAL, "moments of %d bits (8 or 32)", bits);
    if (!d_hyper && !h_hyper) return fail(CHIMERA_EINVAL, "hyperparameters are NULL");
    if ((uintptr_t)d_hyper & 15) return fail(CHIMERA_EINVAL, "device hyperparameters must be 16-byte aligned");
    return d_hyper ? CHIMERA_OK : check_hyper(*h_hyper);
}

}  // namespace chimera

using namespace chimera;

#define STEP_TRY(expr) do { int rc__ = (expr); if (rc__) return rc__; } while (0)

extern "C" {

size_t chimera_op_grad_norm_workspace_bytes(int count) { return count < 1 ? 0 : norm_bytes(count); }

int chimera_op_grad_norm(int count, const int64_t* h_n, const float* const* h_grad, float max_norm, float* d_out, void* d_workspace, size_t workspace_bytes,
                         void* hip_stream) {
    if (count < 1 || !h_n || !h_grad) return fail(CHIMERA_EINVAL, "no tensors");
    if (!d_out || !d_workspace) return fail(CHIMERA_EINVAL, "NULL operand");
    if (!(max_norm > 0)) return fail(CHIMERA_EINVAL, "max_norm must be positive");
    if (((uintptr_t)d_workspace & 7) || ((uintptr_t)d_out & 3)) return fail(CHIMERA_EINVAL, "workspace must be 8-byte aligned, the result 4-byte aligned");
    long long chunk;
    if (!norm_chunk(count, h_n, chunk)) return fail(CHIMERA_EINVAL, "a tensor's size is negative, or the tensors are too large");
    for (int i = 0; i < count; ++i)
        if (h_n[i] && (!h_grad[i] || ((uintptr_t)h_grad[i] & 3))) return fail(CHIMERA_EINVAL, "gradient %d is NULL or not aligned to floats", i);
    if (workspace_bytes < norm_bytes(count)) return fail(CHIMERA_ENOMEM, "workspace holds %zu bytes, need %zu", workspace_bytes, norm_bytes(count));
    const Span out{(uintptr_t)d_out, (uintptr_t)d_out + 8}, rest{(uintptr_t)d_workspace, (uintptr_t)d_workspace + norm_bytes(count)};
    auto meet = [](const Span& a, const Span& b) { return a.begin < b.end && b.begin < a.end; };
    bool apart = !meet(out, rest);
    for (int i = 0; i < count; ++i) {
        const Span g{(uintptr_t)h_grad[i], (uintptr_t)h_grad[i] + (size_t)h_n[i] * 4};
        apart = apart && !(h_n[i] && (meet(g, out) || meet(g, rest)));
    }
    if (!apart) return fail(CHIMERA_EINVAL, "the result or the workspace overlaps a gradient, or one another");
    hipStream_t s = (hipStream_t)hip_stream;
    NormLaunch L{};
    L.chunk = chunk;
    long long done = 0;
    for (int i = 0; i < count;) {
        std::fill(std::begin(L.first), std::end(L.first), INT_MAX);
        long long chunks = 0;
        int used = 0;
        for (; i < count && used < NORM_TENSORS; ++i) {
            if (!h_n[i]) continue;
            L.g[used] = h_grad[i]; L.n[used] = h_n[i]; L.first[used++] = (int)chunks;
            chunks += (h_n[i] + chunk - 1) / chunk;
        }
        if (!used) continue;
        L.partial = (double*)d_workspace + done;
        hipLaunchKernelGGL(grad_square_kernel, dim3((unsigned)chunks), dim3(STEP_THREADS), 0, s, L);
        CHIMERA_LAUNCH_CHECK("gradient norm");
        done += chunks;
    }
    hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(1024), 0, s, (const double*)d_workspace, (int)done, max_norm, d_out);
    CHIMERA_LAUNCH_CHECK("gradient norm");
    return CHIMERA_OK;
}

int chimera_op_adamw(int dtype, int state_bits, int count, const int64_t* h_n, void* const* h_param, float* const* h_master, const float* const* h_grad,
                     void* const* h_m, void* const* h_v, float* const* h_scale, const float* h_decay, const chimera_adamw_hyper* h_hyper, void* d_hyper,
                     const float* d_grad_scale, void* hip_stream) {
    STEP_TRY(adamw_check(dtype, state_bits, h_hyper, d_hyper));
    if (count < 1 || !h_n || !h_param || !h_grad || !h_m || !h_v) return fail(CHIMERA_EINVAL, "no tensors");
    if (dtype == CHIMERA_BF16 && !h_master) return fail(CHIMERA_EINVAL, "bf16 weights need float master weights");
    if (state_bits == 8 && !h_scale) return fail(CHIMERA_EINVAL, "8-bit moments need scales");
    const size_t e = dtype == CHIMERA_F32 ? 4 : 2;
    try {
        std::vector<AdamwTensor> t((size_t)count);
        Spans<7> spans((size_t)count + 1);                                    // weights, master weights, moments, scales, hyperparameters; what is read
        for (int i = 0; i < count; ++i) {
            if (h_n[i] < 0 || h_n[i] > 1ll << 32) return fail(CHIMERA_EINVAL, "tensor %d of %lld values", i, (long long)h_n[i]);
            t[i] = {h_param[i], h_m[i], h_v[i], dtype == CHIMERA_BF16 ? h_master[i] : nullptr, state_bits == 8 ? h_scale[i] : nullptr, h_grad[i], h_n[i],
                    h_decay ? h_decay[i] : 0.f};
            if (!h_n[i]) continue;
            const AdamwTensor& q = t[i];
            if (!q.p || !q.m || !q.v || !q.g || (dtype == CHIMERA_BF16 && !q.master) || (state_bits == 8 && !q.scale)) return fail(CHIMERA_EINVAL, "NULL operand in tensor %d", i);
            if (((uintptr_t)q.p & (e - 1)) || (((uintptr_t)q.master | (uintptr_t)q.g | (uintptr_t)q.scale) & 3) ||
                (state_bits == 32 && (((uintptr_t)q.m | (uintptr_t)q.v) & 3)))
                return fail(CHIMERA_EINVAL, "tensor %d is not aligned to its elements", i);
            if (!(q.decay >= 0) || !std::isfinite(q.decay)) return fail(CHIMERA_EINVAL, "weight decay of tensor %d must be finite and not negative", i);
            const size_t moment = (size_t)h_n[i] * (state_bits == 32 ? 4 : 1);
            spans.add(0, q.p, (size_t)h_n[i] * e);
            spans.add(1, q.master, (size_t)h_n[i] * 4);
            spans.add(2, q.m, moment);
            spans.add(3, q.v, moment);
            spans.add(4, q.scale, (size_t)(h_n[i] + MOMENT_BLOCK - 1) / MOMENT_BLOCK * 8);
            spans.add(6, q.g, (size_t)h_n[i] * 4);
        }
        spans.add(5, d_hyper, CHIMERA_ADAMW_HYPER_BYTES);
        spans.add(6, d_grad_scale, 4);
        if (spans.written_twice()) return fail(CHIMERA_EINVAL, "what the step writes overlaps: weights, master weights, moments, scales, hyperparameters, or a gradient or factor with one of these");
        return adamw_step(dtype, state_bits, count, t.data(), h_hyper, d_hyper, d_grad_scale, hip_stream);
    } catch (const std::bad_alloc&) {
        return fail(CHIMERA_ENOMEM, "out of host memory");
    }
}

}  // extern "C"
