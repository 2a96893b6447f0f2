// Orthogonalisation of updates by Newton-Schulz products.
//
// X0 = G / (|G| + eps);  X <- a X + (b A + c A A) X, A = X X^T, on the shorter
// side s of the matrix (L the longer).  Every X is Q X0 with Q a polynomial of
// A0 = X0 X0^T, and all these polynomials commute and are symmetric, so a step is
//   P = a I + b A + c A A,  Q <- P Q,  A <- P A P
// on s x s matrices, and the long side is touched twice: A0 and Q X0.
#include <math.h>

#include <algorithm>

#include "sb_common.h"
#include "sb_kernels.h"

namespace sb {

namespace {

// One matrix: X [s][L] (the update, transposed if it is tall, times the power
// of two that brings its largest value to [1, 2)).
struct View {
    long long ld;
    int s, L;
    bool tall;
};

constexpr int OT = 64;  // tile side of the products

__device__ __forceinline__ float pow2_scale(float amax) {
    int e = 0;
    if (amax > 0.0f && amax < INFINITY) frexpf(amax, &e);
    return ldexpf(1.0f, max(-100, min(100, 1 - e)));
}

template <typename T>
__global__ __launch_bounds__(1024) void k_amax(const T* g, View v, float* scal) {
    __shared__ float s[16];
    float m = 0.0f;
    const int rows = v.tall ? v.L : v.s, cols = v.tall ? v.s : v.L;
    for (int r = 0; r < rows; ++r)
        for (int c = (int)threadIdx.x; c < cols; c += 1024) m = fmaxf(m, fabsf(to_f32(g[r * v.ld + c])));
    for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
    if (lane_id() == 0) s[threadIdx.x >> 6] = m;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 16; ++w) m = fmaxf(m, s[w]);
        scal[0] = pow2_scale(m);
    }
}

template <typename T>
__global__ __launch_bounds__(WG) void k_scaled(const T* g, View v, const float* scal, float* X) {
    const float f = scal[0];
    const int i = (int)blockIdx.y;
    const int k = (int)(blockIdx.x * WG + threadIdx.x);
    if (k < v.L) X[(size_t)i * v.L + k] = to_f32(v.tall ? g[k * v.ld + i] : g[i * v.ld + k]) * f;
}

// C = alpha A B^T + beta D + gamma I of [M][K] and [N][K], K-contiguous (BT: B is [K][N]).
template <bool BT, typename TO>
__global__ __launch_bounds__(WG) void k_product(const float* A, const float* B, int M, int N, int K, float alpha,
                                                const float* D, float beta, float gamma, const float* scal, TO* C,
                                                long long ldc, bool ct) {
    __shared__ float sa[16][OT + 1], sb[16][OT + 1];
    const int i0 = (int)blockIdx.y * OT, j0 = (int)blockIdx.x * OT, tid = (int)threadIdx.x;
    const int ti = tid >> 4, tj = tid & 15;
    float acc[4][4] = {};
    for (int k0 = 0; k0 < K; k0 += 16) {
        for (int e = tid; e < OT * 16; e += WG) {
            const int r = e >> 4, k = e & 15, rb = BT ? e & 63 : r, kb = BT ? e >> 6 : k;
            sa[k][r] = i0 + r < M && k0 + k < K ? A[(size_t)(i0 + r) * K + k0 + k] : 0.0f;
            sb[kb][rb] = j0 + rb < N && k0 + kb < K
                             ? (BT ? B[(size_t)(k0 + kb) * N + j0 + rb] : B[(size_t)(j0 + rb) * K + k0 + kb])
                             : 0.0f;
        }
        __syncthreads();
        for (int k = 0; k < 16; ++k)
            for (int x = 0; x < 4; ++x)
                for (int y = 0; y < 4; ++y) acc[x][y] += sa[k][ti * 4 + x] * sb[k][tj * 4 + y];
        __syncthreads();
    }
    const float f = scal ? alpha * scal[1] : alpha;
    for (int x = 0; x < 4; ++x)
        for (int y = 0; y < 4; ++y) {
            const int i = i0 + ti * 4 + x, j = j0 + tj * 4 + y;
            if (i >= M || j >= N) continue;
            float r = f * acc[x][y] + (i == j ? gamma : 0.0f);
            if (D) r += beta * D[(size_t)i * N + j];
            C[ct ? j * ldc + i : i * ldc + j] = from_f32<TO>(r);
        }
}

// scal[1] = 1 / (|X| + eps scale) from the trace of X X^T, and A0 = X X^T scal[1]^2.
__global__ __launch_bounds__(WG) void k_norm(const float* A, int s, float eps, float* scal) {
    __shared__ float w[WG / 64];
    float t = 0.0f;
    for (int i = (int)threadIdx.x; i < s; i += WG) t += A[(size_t)i * s + i];
    for (int o = 32; o > 0; o >>= 1) t += __shfl_xor(t, o, 64);
    if (lane_id() == 0) w[threadIdx.x >> 6] = t;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int k = 1; k < WG / 64; ++k) t += w[k];
        scal[1] = t == 0.0f ? 0.0f : t < INFINITY ? 1.0f / (sqrtf(t) + eps * scal[0]) : NAN;
    }
}
__global__ __launch_bounds__(WG) void k_normalise(float* A, long long n, const float* scal) {
    const long long i = (long long)blockIdx.x * WG + threadIdx.x;
    if (i < n) A[i] = A[i] * scal[1] * scal[1];
}
__global__ __launch_bounds__(WG) void k_identity(float* Q, int s) {
    const long long i = (long long)blockIdx.x * WG + threadIdx.x;
    if (i < (long long)s * s) Q[i] = i / s == i % s ? 1.0f : 0.0f;
}

size_t up256(size_t b) { return (b + 255) / 256 * 256; }

size_t one_bytes(const OrthMat& q) {
    const size_t s = (size_t)std::min(q.m, q.n), L = (size_t)std::max(q.m, q.n);
    return 256 + up256(s * L * 4) + 5 * up256(s * s * 4);
}

template <typename T>
hipError_t orth_one(const T* g, T* o, const OrthMat& q, int steps, const double* coef, double eps, char* ws,
                    hipStream_t st) {
    const bool tall = q.m > q.n;
    const int s = std::min(q.m, q.n), L = std::max(q.m, q.n);
    const View v{q.ld, s, L, tall};
    float* scal = (float*)ws;
    float* X = (float*)(ws + 256);
    float* mat[5];
    char* at = ws + 256 + up256((size_t)s * L * 4);
    for (int i = 0; i < 5; ++i, at += up256((size_t)s * s * 4)) mat[i] = (float*)at;
    float *A = mat[0], *P = mat[1], *Tm = mat[2], *Q = mat[3], *Q2 = mat[4];
    hipLaunchKernelGGL(k_amax<T>, dim3(1), dim3(1024), 0, st, g, v, scal);
    hipLaunchKernelGGL(k_scaled<T>, dim3((L + WG - 1) / WG, s), dim3(WG), 0, st, g, v, (const float*)scal, X);
    const dim3 sq((s + OT - 1) / OT, (s + OT - 1) / OT);
    const unsigned flat = (unsigned)(((long long)s * s + WG - 1) / WG);
    auto mul = [&](const float* a, const float* b, float* c, float alpha, const float* d, float beta, float gamma) {
        hipLaunchKernelGGL((k_product<false, float>), sq, dim3(WG), 0, st, a, b, s, s, s, alpha, d, beta, gamma,
                           (const float*)nullptr, c, (long long)s, false);
    };
    hipLaunchKernelGGL((k_product<false, float>), sq, dim3(WG), 0, st, (const float*)X, (const float*)X, s, s, L, 1.0f,
                       (const float*)nullptr, 0.0f, 0.0f, (const float*)nullptr, A, (long long)s, false);
    hipLaunchKernelGGL(k_norm, dim3(1), dim3(WG), 0, st, (const float*)A, s, (float)eps, scal);
    hipLaunchKernelGGL(k_normalise, dim3(flat), dim3(WG), 0, st, A, (long long)s * s, (const float*)scal);
    hipLaunchKernelGGL(k_identity, dim3(flat), dim3(WG), 0, st, Q, s);
    for (int i = 0; i < steps; ++i) {
        const float a = (float)coef[3 * i], b = (float)coef[3 * i + 1], c = (float)coef[3 * i + 2];
        mul(A, A, P, c, A, b, a);
        mul(P, Q, Q2, 1.0f, nullptr, 0.0f, 0.0f);
        std::swap(Q, Q2);
        if (i + 1 == steps) break;
        mul(P, A, Tm, 1.0f, nullptr, 0.0f, 0.0f);
        mul(Tm, P, A, 1.0f, nullptr, 0.0f, 0.0f);
    }
    hipLaunchKernelGGL((k_product<true, T>), dim3((L + OT - 1) / OT, (s + OT - 1) / OT), dim3(WG), 0, st,
                       (const float*)Q, (const float*)X, s, L, s, 1.0f, (const float*)nullptr, 0.0f, 0.0f,
                       (const float*)scal, o, q.ld_o, tall);
    return hipGetLastError();
}

template <typename T>
hipError_t orth_t(const OrthMat* mats, int count, int steps, const double* coef, double eps, Ws ws, hipStream_t st) {
    for (int i = 0; i < count; ++i)
        for (int b = 0; b < mats[i].batch; ++b) {
            const hipError_t e = orth_one<T>((const T*)mats[i].g + b * mats[i].bstride, (T*)mats[i].o + b * mats[i].bstride_o,
                                             mats[i], steps, coef, eps, (char*)ws.p, st);
            if (e != hipSuccess) return e;
        }
    return hipSuccess;
}

}  // namespace

size_t orth_ws_bytes(int, const OrthMat* mats, int count) {
    size_t n = 0;
    for (int i = 0; i < count; ++i) n = std::max(n, one_bytes(mats[i]));
    return n;
}

hipError_t launch_orth(int dtype, const OrthMat* mats, int count, int steps, const double* coef, double eps, Ws ws,
                       hipStream_t st) {
    if (dtype == 0) return orth_t<float>(mats, count, steps, coef, eps, ws, st);
    if (dtype == 1) return orth_t<f16>(mats, count, steps, coef, eps, ws, st);
    return orth_t<bf16>(mats, count, steps, coef, eps, ws, st);
}

}  // namespace sb
