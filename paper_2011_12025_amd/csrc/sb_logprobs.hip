// Log probabilities of class scores, and their gradient.
//
// A row is a pixel's (or token's) C scores z.  With m = max z, e_j = exp(z_j - m),
// s = sum e_j and t = sum e_j (z_j - m):
//   lse = m + ln s,  logp = (z_label - m) - ln s,  entropy = ln s - t / s.
// The running (m, s, t) of a part of a row is rescaled when its maximum grows,
// so a row is read once; two parts join by the same rule.  All of it is fp32.
// exp is 2^((z - m) log2 e) with the difference taken first: scores as low as
// the type allows, in all classes of a row, still give a uniform row.
//
// Gradient, with p_j = exp(z_j - lse) and G the sum of the row's gradients of
// log probabilities:
//   dz_j = [j = label] g + sum_i [j = top_i] g_i - p_j (G + g_H (ln p_j + H)).
#include <math.h>

#include "sb_common.h"
#include "sb_kernels.h"

namespace sb {

namespace {

typedef unsigned long long u64;

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float LOWEST = -3.402823466e38f;  // below every score that is not -inf
constexpr float FAR = -1000.0f;             // 2^FAR is 0; keeps 0 * -inf out of t

struct Acc {
    float m, s, t;  // t in units of log2
};
__device__ __forceinline__ Acc nothing() { return Acc{LOWEST, 0.0f, 0.0f}; }

__device__ __forceinline__ float exp2_(float v) { return __builtin_amdgcn_exp2f(v); }

// (m, s, t) brought to the maximum m2 >= m.
__device__ __forceinline__ void raise(Acc& a, float m2) {
    const float d = fmaxf((a.m - m2) * LOG2E, FAR), e = exp2_(d);
    a.t = (a.t + a.s * d) * e;
    a.s *= e;
    a.m = m2;
}

__device__ __forceinline__ void join(Acc& a, Acc b) {
    const float m = fmaxf(a.m, b.m);
    raise(a, m);
    raise(b, m);
    a.s += b.s;
    a.t += b.t;
}

__device__ __forceinline__ void add(Acc& a, float z) {
    if (z > a.m) raise(a, z);
    const float d = (z - a.m) * LOG2E, e = exp2_(d);  // (NaN stays in e)
    a.s += e;
    a.t += e * fmaxf(d, FAR);
}

__device__ __forceinline__ Acc wave_join(Acc a) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        Acc b;
        b.m = __shfl_xor(a.m, o, 64);
        b.s = __shfl_xor(a.s, o, 64);
        b.t = __shfl_xor(a.t, o, 64);
        join(a, b);
    }
    return a;
}

// Order of the alternatives as one integer: the larger score, then the lower
// class.  -0 counts as 0, NaN as the largest; 0 is below every class.
__device__ __forceinline__ u64 key_of(float z, int j) {
    uint32_t b = __float_as_uint(z + 0.0f);
    b = z != z ? 0xFFFFFFFFu : (b & 0x80000000u) ? ~b : b | 0x80000000u;
    return (u64)b << 32 | (uint32_t)~j;
}
__device__ __forceinline__ int key_class(u64 k) { return (int)~(uint32_t)k; }
__device__ __forceinline__ float key_score(u64 k) {
    const uint32_t b = (uint32_t)(k >> 32);
    return __uint_as_float(b == 0xFFFFFFFFu ? 0x7FC00000u : (b & 0x80000000u) ? b ^ 0x80000000u : ~b);
}

struct Row {
    float m, ln_s;  // s = 0 (every class at -inf): an empty row
    bool empty;
    __device__ __forceinline__ explicit Row(const Acc& a) : m(a.m), ln_s(logf(a.s)), empty(a.s == 0.0f) {}
    __device__ __forceinline__ float logp(float z) const { return empty ? -INFINITY : (z - m) - ln_s; }
    __device__ __forceinline__ float lse() const { return empty ? -INFINITY : m + ln_s; }
    __device__ __forceinline__ float entropy(const Acc& a) const { return empty ? 0.0f : ln_s - LN2 * a.t / a.s; }
};

// One 256-thread workgroup a row, class by class; the alternatives one after
// the other, each the largest key below the one before.
template <typename T>
__global__ __launch_bounds__(WG) void k_logp_row(LogpArgs a) {
    const long long r = blockIdx.x, n = r / a.P, p = r - n * a.P;
    const T* z = (const T*)a.z + n * a.C_buf * a.P + p;
    __shared__ Acc s_acc[WG / 64];
    __shared__ u64 s_key[WG / 64];
    const int tid = (int)threadIdx.x, lane = lane_id(), wave = tid >> 6;
    Acc acc = nothing();
    for (int j = tid; j < a.C; j += WG) add(acc, to_f32(z[j * a.P]));
    acc = wave_join(acc);
    if (lane == 0) s_acc[wave] = acc;
    __syncthreads();
    acc = s_acc[0];
    for (int w = 1; w < WG / 64; ++w) join(acc, s_acc[w]);
    const Row row(acc);
    if (tid == 0) {
        a.lse[r] = row.lse();
        if (a.entropy) a.entropy[r] = row.entropy(acc);
        if (a.labels) {
            const long long t = a.labels[r];
            a.logp[r] = t == a.ignore ? 0.0f : t < 0 || t >= a.C ? NAN : row.logp(to_f32(z[t * a.P]));
        }
    }
    u64 last = ~0ull;
    for (int i = 0; i < a.topk; ++i) {
        u64 best = 0;
        for (int j = tid; j < a.C; j += WG) {
            const u64 k = key_of(to_f32(z[j * a.P]), j);
            if (k < last && k > best) best = k;
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            const u64 k = __shfl_xor(best, o, 64);
            best = k > best ? k : best;
        }
        __syncthreads();
        if (lane == 0) s_key[wave] = best;
        __syncthreads();
        for (int w = 0; w < WG / 64; ++w) best = s_key[w] > best ? s_key[w] : best;
        if (tid == 0) {
            const long long q = (n * a.topk + i) * a.P + p;
            a.top_logp[q] = row.logp(key_score(best));
            a.top_index[q] = key_class(best);
        }
        last = best;
    }
}

template <typename T>
__global__ __launch_bounds__(WG) void k_logp_grad_row(LogpGradArgs a) {
    const long long r = blockIdx.x, n = r / a.P, p = r - n * a.P;
    const T* z = (const T*)a.z + n * a.C_buf * a.P + p;
    T* dz = (T*)a.dz + n * a.C_dbuf * a.P + p;
    float lse = a.lse[r], g = 0.0f;
    long long label = -1;
    if (a.d_logp) {
        label = a.labels[r];
        if (label == a.ignore) label = -1;
        else g = label < 0 || label >= a.C ? NAN : a.d_logp[r];
    }
    const float gh = a.d_entropy ? a.d_entropy[r] : 0.0f, H = a.d_entropy ? a.entropy[r] : 0.0f;
    auto top = [&](int i) { return (n * a.topk + i) * a.P + p; };
    float G = g;
    for (int i = 0; i < a.topk; ++i) {
        const int j = a.top_index[top(i)];
        G += j < 0 || j >= a.C ? NAN : a.d_top[top(i)];
    }
    // p from lse is off by |lse| 2^-25: past 256 it comes from the row's own maximum
    float m = lse, ln_s = 0.0f;
    if (fabsf(lse) > 256.0f && lse != -INFINITY) {
        Acc acc = nothing();
        for (int j = 0; j < a.C; ++j) add(acc, to_f32(z[j * a.P]));
        const Row row(acc);
        m = row.m;
        ln_s = row.ln_s;
    }
    for (int j = (int)threadIdx.x; j < a.C; j += WG) {
        const float lp = (to_f32(z[j * a.P]) - m) - ln_s, pr = exp2_(lp * LOG2E);
        float d = -pr * (G + gh * (fmaxf(lp, FAR) + H));
        if (j == label) d += g;
        for (int i = 0; i < a.topk; ++i)
            if (a.top_index[top(i)] == j) d += a.d_top[top(i)];
        dz[j * a.P] = from_f32<T>(lse == -INFINITY ? 0.0f : d);
    }
}

}  // namespace

int logp_max_top() { return 64; }

size_t logp_ws_bytes(int, const LogpArgs&) { return 0; }

hipError_t launch_logp(int dtype, const LogpArgs& a, Ws, hipStream_t st) {
    const dim3 grid((unsigned)a.R), block(WG);
    if (dtype == 0) hipLaunchKernelGGL(k_logp_row<float>, grid, block, 0, st, a);
    else if (dtype == 1) hipLaunchKernelGGL(k_logp_row<f16>, grid, block, 0, st, a);
    else hipLaunchKernelGGL(k_logp_row<bf16>, grid, block, 0, st, a);
    return hipGetLastError();
}

hipError_t launch_logp_grad(int dtype, const LogpGradArgs& a, hipStream_t st) {
    const dim3 grid((unsigned)a.R), block(WG);
    if (dtype == 0) hipLaunchKernelGGL(k_logp_grad_row<float>, grid, block, 0, st, a);
    else if (dtype == 1) hipLaunchKernelGGL(k_logp_grad_row<f16>, grid, block, 0, st, a);
    else hipLaunchKernelGGL(k_logp_grad_row<bf16>, grid, block, 0, st, a);
    return hipGetLastError();
}

}  // namespace sb
