// Orthogonalisation of updates by Newton-Schulz products.
//
// X0 = G / (|G| + eps);  X <- a X + (b A + c A A) X, A = X X^T, on the shorter
// side s of the matrix (L the longer).  After several steps X is Q X0 with Q a
// polynomial of A0 = X0 X0^T; these polynomials commute and are symmetric, so
// a step is
//   P = a I + b A + c A A,  Q <- P Q,  A <- P A P
// on s x s matrices (symmetric products: half of the tiles), and the long side
// is touched twice for a block of steps: A0 and Q X0.
//
// Precision.  An error of A grows by p(0)^2 = a^2 (11.9) a step in the
// directions of small singular values, whatever the spectrum, because there
// A <- P A P multiplies by it.  So a block ends when that growth would show in
// the result (MAX_GROWTH) and the next one starts from a fresh X X^T: five
// steps are blocks of 3 and 2 for fp32 and fp16, where the error is that of an
// fp32 iteration (2.7e-6 of the norm against 2.1e-6 at 350 x 1500), and one
// block for bf16 (2e-4, a tenth of its rounding).  All s x s matrices and all
// X but the first are pairs of fp16 numbers hi + lo (22 bits and a sign) times
// a power of two known beforehand from the polynomial's bounds; a product of
// two is three MFMAs hi hi + hi lo + lo hi with fp32 sums.  The first X is one
// fp16 number for 16-bit updates (their values times a power of two; bf16
// values below 2^-38 of the largest are cut) and a pair for fp32.
#include <math.h>

#include <algorithm>
#include <type_traits>
#include <vector>

#include "sb_common.h"
#include "sb_kernels.h"

namespace sb {

namespace {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef _Float16 halfx8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) void* lds_ptr;

// ---------------------------------------------------------------------------
// What a launch works on: up to OM entries of the list, each a batch of equal
// matrices, blocks numbered entry by entry (start).
// ---------------------------------------------------------------------------
constexpr int OM = 30;  // (the table is a kernel argument, at most 4 KB)

struct OMat {
    const void* g;
    void* o;
    long long ld, ld_o, bstride, bstride_o;
    char* ws;        // of the first matrix; the next one's is ws_one bytes on
    long long ws_one;
    int batch, m, n, s, L, sp, Lp;  // sp, Lp: s, L rounded up to whole tiles (zeros)
    int splits;                     // of the product over L
};
struct Table {
    OMat mat[OM];
    int start[OM + 1];
    int count;
};

// The workspace of one matrix, in bytes from its start.
constexpr int MAXP = 1024;  // workgroups that make X, each with its sum of squares
constexpr int MAXA = 256;   // workgroups that look for the largest value
constexpr long long W_SUM = 1024, W_X = W_SUM + 4 * MAXP;  // [0]: the largest values
__host__ __device__ inline long long w_x_bytes(int sp, int Lp) { return (long long)sp * Lp * 4; }
__host__ __device__ inline long long w_xt(int sp, int Lp, int i) { return W_X + (1 + i) * w_x_bytes(sp, Lp); }
__host__ __device__ inline long long w_sym(int sp, int Lp, int i) {
    return W_X + 3 * w_x_bytes(sp, Lp) + i * ((long long)sp * sp * 4);
}
constexpr int SYMS = 5;  // A, T and three that P and Q take in turn

struct Place {  // of a workgroup
    int mat, b, t;  // entry, matrix of its batch, tile
};
template <typename F>  // per_of: workgroups of one matrix of an entry
__device__ __forceinline__ Place place(const Table& tb, F per_of) {
    const int bid = (int)blockIdx.x, l = lane_id();
    const int i = __popcll(__ballot(l < tb.count && bid >= tb.start[min(l, OM)])) - 1;
    const int t = bid - tb.start[i], per = per_of(tb.mat[i]);
    return Place{i, t / per, t % per};
}

__device__ __forceinline__ int amax_wgs(const OMat& q) {
    return (int)min((long long)MAXA, ((long long)q.m * q.n + 16383) / 16384);
}
__device__ __forceinline__ int prep_wgs(const OMat& q) {
    return (int)min((long long)MAXP, (long long)(q.sp / 64) * (q.Lp / 64));
}

// ---------------------------------------------------------------------------
// Storage of a matrix of pairs: a row is [k / 32][32 hi | 32 lo]; of single
// numbers: [k].  NP: numbers an element.
// ---------------------------------------------------------------------------
template <int NP>
__device__ __forceinline__ long long at_k(long long k) {  // bytes, k a multiple of 8
    return NP == 2 ? (k >> 5) * 128 + (k & 31) * 2 : k * 2;
}

template <int NP>
__device__ __forceinline__ void store8(char* row, long long k, const float (&v)[8]) {
    Vec<f16, 8> hi, lo;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        // Kept apart from the multiplication that gave it: the compiler otherwise
        // takes hi for the store from v_cvt_pk_f16_f32 of the rounded product and
        // hi for the difference from v_fma_mixlo_f16, which rounds once; where the
        // two differ lo belongs to the other one.
        float x = v[i];
        asm("" : "+v"(x));
        hi.e[i] = (f16)x;
        lo.e[i] = (f16)(x - (float)hi.e[i]);
    }
    char* p = row + at_k<NP>(k);
    vstore<f16, 8>((f16*)p, hi);
    if (NP == 2) vstore<f16, 8>((f16*)(p + 64), lo);
}

// A T x T tile in LDS (fp32, rows CP<T> apart) to rows r0.. and columns c0.. of a
// matrix with K columns; turned: its transpose.
template <int T> constexpr int CP = T + 1;

template <int T, int NP>
__device__ __forceinline__ void store_tile(const float* C, char* dst, long long K, int r0, int c0, bool turned) {
    for (int e = (int)threadIdx.x; e < T * T / 8; e += WG) {
        const int r = e / (T / 8), k = (e % (T / 8)) * 8;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = turned ? C[(k + i) * CP<T> + r] : C[r * CP<T> + k + i];
        store8<NP>(dst + (long long)(r0 + r) * K * (2 * NP), c0 + k, v);
    }
}

// ---------------------------------------------------------------------------
// The first X.
// ---------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(WG) void k_orth_amax(Table tb) {
    __shared__ float s[WG / 64];
    const Place p = place(tb, [](const OMat& q) { return amax_wgs(q); });
    const OMat& q = tb.mat[p.mat];
    const T* g = (const T*)q.g + p.b * q.bstride;
    const int wave = (int)threadIdx.x >> 6, l = lane_id(), all = amax_wgs(q) * (WG / 64);
    float m = 0.0f;
    for (int r = p.t * (WG / 64) + wave; r < q.m; r += all)
        for (int c = l; c < q.n; c += 64) m = fmaxf(m, fabsf(to_f32(g[r * q.ld + c])));
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
    if (l == 0) s[wave] = m;
    __syncthreads();
    if (threadIdx.x == 0) ((float*)(q.ws + p.b * q.ws_one))[p.t] = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
}

// The sum of n floats (fixed order) or their maximum, over a workgroup.
template <bool MAX>
__device__ __forceinline__ float wg_reduce(const float* p, int n, float* s4) {
    float v = 0.0f;
    for (int i = (int)threadIdx.x; i < n; i += WG) v = MAX ? fmaxf(v, p[i]) : v + p[i];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const float w = __shfl_xor(v, o, 64);
        v = MAX ? fmaxf(v, w) : v + w;
    }
    __syncthreads();
    if (lane_id() == 0) s4[threadIdx.x >> 6] = v;
    __syncthreads();
    return MAX ? fmaxf(fmaxf(s4[0], s4[1]), fmaxf(s4[2], s4[3])) : (s4[0] + s4[1]) + (s4[2] + s4[3]);
}

// The power of two that brings the largest value to [2^13, 2^14).
__device__ __forceinline__ int scale_of(const OMat& q, const char* ws, float* s4) {
    const float m = wg_reduce<true>((const float*)ws, amax_wgs(q), s4);
    int e = 0;
    if (m > 0.0f && m < INFINITY) frexpf(m, &e);
    return max(-126, min(126, m > 0.0f ? 14 - e : 0));
}

// 1 / (|G| + eps) for X as it is stored: 0 for zeros, NaN where |G| is not finite.
__device__ __forceinline__ float norm_factor(const OMat& q, const char* ws, float eps, float* s4) {
    const int e = scale_of(q, ws, s4);
    const float t = wg_reduce<false>((const float*)(ws + W_SUM), prep_wgs(q), s4);
    return t == 0.0f ? 0.0f : t < INFINITY ? 1.0f / (sqrtf(t) + ldexpf(eps, e)) : NAN;
}

// X [sp][Lp] and its transpose [Lp][sp] from the update, and its squares.
template <typename T>
__global__ __launch_bounds__(WG) void k_orth_prep(Table tb) {
    constexpr int NP = sizeof(T) == 4 ? 2 : 1;
    __shared__ float C[64 * CP<64>];
    __shared__ float s4[WG / 64];
    const Place p = place(tb, [](const OMat& q) { return prep_wgs(q); });
    const OMat& q = tb.mat[p.mat];
    const T* g = (const T*)q.g + p.b * q.bstride;
    char* ws = q.ws + p.b * q.ws_one;
    const int e = scale_of(q, ws, s4), tid = (int)threadIdx.x;
    const bool tall = q.m > q.n;
    const int mp = tall ? q.Lp : q.sp, np = tall ? q.sp : q.Lp, tn = np / 64, tiles = (mp / 64) * tn, wgs = prep_wgs(q);
    char* X = ws + W_X;                     // [sp][Lp]
    char* Xt = ws + w_xt(q.sp, q.Lp, 0);    // [Lp][sp]
    float sum = 0.0f;
    for (int t = p.t; t < tiles; t += wgs) {
        const int r0 = t / tn * 64, c0 = t % tn * 64;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int r = r0 + i * 4 + (tid >> 6), c = c0 + (tid & 63);
            const float v = r < q.m && c < q.n ? ldexpf(to_f32(g[r * q.ld + c]), e) : 0.0f;
            C[(i * 4 + (tid >> 6)) * CP<64> + (tid & 63)] = v;
            sum += v * v;
        }
        __syncthreads();
        store_tile<64, NP>(C, tall ? Xt : X, np, r0, c0, false);
        store_tile<64, NP>(C, tall ? X : Xt, mp, c0, r0, true);
        __syncthreads();
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
    if (lane_id() == 0) s4[tid >> 6] = sum;
    __syncthreads();
    if (tid == 0) ((float*)(ws + W_SUM))[p.t] = (s4[0] + s4[1]) + (s4[2] + s4[3]);
}

// ---------------------------------------------------------------------------
// A T x T tile of A B^T, K in steps of 32: both operands' rows go to LDS by DMA
// (16 bytes a lane) while the step before is multiplied.  128 (64) bytes a row
// and step, its 16-byte chunks XORed by the row, so that the rows which an MFMA
// operand reads together lie in distinct banks.  Four waves, each a quarter of
// the tile in v_mfma_f32_32x32x16_f16.
// ---------------------------------------------------------------------------
template <int T> constexpr int MF = T / 64;  // 32 x 32 fragments of a wave, each way

template <int NP>
__device__ __forceinline__ int chunk_of(int row, int c) {  // where chunk c of a row lies
    return NP == 2 ? c ^ (row & 7) : c ^ ((row >> 1) & 3);
}

template <int T, int NP>
__device__ __forceinline__ void stage(const char* rows, long long pitch, int step, unsigned char* lds) {
    const int tid = (int)threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
#pragma unroll
    for (int i = 0; i < T * 4 * NP / WG; ++i) {
        const int c = i * WG + tid, r = c / (4 * NP);
        const char* src = rows + r * pitch + (long long)step * (64 * NP) + chunk_of<NP>(r, c % (4 * NP)) * 16;
        __builtin_amdgcn_global_load_lds(src, (lds_ptr)(lds + (i * WG + wave * 64) * 16), 16, 0, 0);
    }
}

template <int T, int NA, int NB> constexpr int stage_bytes() { return T * 64 * (NA + NB); }
template <int T, int NA, int NB> constexpr int product_lds() {
    return std::max(2 * stage_bytes<T, NA, NB>(), T * CP<T> * 4);
}

__device__ __forceinline__ void product_barrier() {  // the DMA before it has landed, for all waves
    __builtin_amdgcn_s_waitcnt(0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// rows of A and B from their first element on; the tile ends in LDS as fp32.
template <int T, int NA, int NB>
__device__ __forceinline__ void product_tile(const char* A, long long pa, const char* B, long long pb, int step0,
                                             int steps, unsigned char* lds) {
    constexpr int SB = stage_bytes<T, NA, NB>(), OB = T * 64 * NA;
    const int l = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int ra = (wave >> 1) * (T / 2) + (l & 31), rb = (wave & 1) * (T / 2) + (l & 31);
    floatx16 acc[MF<T>][MF<T>] = {};
    stage<T, NA>(A, pa, step0, lds);
    stage<T, NB>(B, pb, step0, lds + OB);
    for (int s = 0; s < steps; ++s) {
        product_barrier();
        unsigned char* cur = lds + (s & 1) * SB;
        if (s + 1 < steps) {
            unsigned char* nxt = lds + (~s & 1) * SB;
            stage<T, NA>(A, pa, step0 + s + 1, nxt);
            stage<T, NB>(B, pb, step0 + s + 1, nxt + OB);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int c = 2 * j + (l >> 5);
            halfx8 fa[NA][MF<T>], fb[NB][MF<T>];
#pragma unroll
            for (int i = 0; i < MF<T>; ++i) {
#pragma unroll
                for (int h = 0; h < NA; ++h)
                    fa[h][i] = *(const halfx8*)(cur + (ra + 32 * i) * (64 * NA) + chunk_of<NA>(ra + 32 * i, 4 * h + c) * 16);
#pragma unroll
                for (int h = 0; h < NB; ++h)
                    fb[h][i] = *(const halfx8*)(cur + OB + (rb + 32 * i) * (64 * NB) +
                                                chunk_of<NB>(rb + 32 * i, 4 * h + c) * 16);
            }
#pragma unroll
            for (int h = 0; h < NA + NB - 1; ++h)  // hi hi, hi lo, lo hi
#pragma unroll
                for (int x = 0; x < MF<T>; ++x)
#pragma unroll
                    for (int y = 0; y < MF<T>; ++y) {
                        const int ha = h == (NB == 2 ? 2 : 1) ? 1 : 0, hb = NB == 2 && h == 1 ? 1 : 0;
                        acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fa[ha < NA ? ha : 0][x], fb[hb < NB ? hb : 0][y],
                                                                           acc[x][y], 0, 0, 0);
                    }
        }
    }
    __syncthreads();
    float* C = (float*)lds;
#pragma unroll
    for (int x = 0; x < MF<T>; ++x)
#pragma unroll
        for (int y = 0; y < MF<T>; ++y)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int i = (wave >> 1) * (T / 2) + 32 * x + (r & 3) + 8 * (r >> 2) + 4 * (l >> 5);
                const int j = (wave & 1) * (T / 2) + 32 * y + (l & 31);
                C[i * CP<T> + j] = acc[x][y][r];
            }
    __syncthreads();
}

template <int T>
__device__ __forceinline__ int sym_tiles(const OMat& q) {
    const int t = q.sp / T;
    return t * (t + 1) / 2;
}
__device__ __forceinline__ void sym_tile(int t, int& bi, int& bj) {  // the t-th tile with bi >= bj
    bi = (int)((sqrtf(8.0f * t + 1.0f) - 1.0f) * 0.5f);
    while ((bi + 1) * (bi + 2) / 2 <= t) ++bi;
    while (bi * (bi + 1) / 2 > t) --bi;
    bj = t - bi * (bi + 1) / 2;
}

// out = alpha C + beta D + gamma I, out and D symmetric [sp][sp], the tile and its mirror image.
template <int T>
__device__ __forceinline__ void store_sym(float* C, char* out, const char* D, int sp, int bi, int bj, float alpha,
                                          float beta, float gamma) {
    for (int e = (int)threadIdx.x; e < T * T / 8; e += WG) {
        const int r = e / (T / 8), k = (e % (T / 8)) * 8, R = bi * T + r, K = bj * T + k;
        const long long row = (long long)R * sp * 4;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = alpha * C[r * CP<T> + k + i];
        if (D) {
            const Vec<f16, 8> hi = vload<f16, 8>((const f16*)(D + row + at_k<2>(K)));
            const Vec<f16, 8> lo = vload<f16, 8>((const f16*)(D + row + at_k<2>(K) + 64));
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += beta * ((float)hi.e[i] + (float)lo.e[i]) + (R == K + i ? gamma : 0.0f);
        }
        store8<2>(out + row, K, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) C[r * CP<T> + k + i] = v[i];
    }
    if (bi == bj) return;
    __syncthreads();
    store_tile<T, 2>(C, out, sp, bj * T, bi * T, true);
}

// A <- X X^T (times norm_factor^2 in the first block) or its parts over K.
template <int T, int NP>
__global__ __launch_bounds__(WG, 2) void k_orth_gram(Table tb, float alpha, float eps, int first) {
    extern __shared__ __align__(16) unsigned char lds[];
    __shared__ float s4[WG / 64];
    // (tile, part): the parts of a tile are neighbours
    const Place p = place(tb, [](const OMat& q) { return sym_tiles<T>(q) * q.splits; });
    const OMat& q = tb.mat[p.mat];
    char* ws = q.ws + p.b * q.ws_one;
    int bi, bj;
    sym_tile(p.t / q.splits, bi, bj);
    const int part = p.t % q.splits, all = q.Lp / 32, k0 = (int)((long long)all * part / q.splits),
              k1 = (int)((long long)all * (part + 1) / q.splits);
    const long long pitch = (long long)q.Lp * (2 * NP);
    const char* X = ws + W_X;
    product_tile<T, NP, NP>(X + bi * T * pitch, pitch, X + bj * T * pitch, pitch, k0, k1 - k0, lds);
    float* C = (float*)lds;
    if (q.splits > 1) {
        float* out = (float*)(ws + w_sym(q.sp, q.Lp, SYMS)) + (long long)p.t * (T * T);
        for (int e = (int)threadIdx.x; e < T * T; e += WG) out[e] = C[e / T * CP<T> + e % T];
        return;
    }
    const float f = first ? norm_factor(q, ws, eps, s4) : 1.0f;
    store_sym<T>(C, ws + w_sym(q.sp, q.Lp, 0), nullptr, q.sp, bi, bj, alpha * f * f, 0.0f, 0.0f);
}

// The parts added in their order.
template <int T>
__global__ __launch_bounds__(WG) void k_orth_parts(Table tb, float alpha, float eps, int first) {
    extern __shared__ __align__(16) unsigned char lds[];
    __shared__ float s4[WG / 64];
    const Place p = place(tb, [](const OMat& q) { return q.splits > 1 ? sym_tiles<T>(q) : 0; });
    const OMat& q = tb.mat[p.mat];
    char* ws = q.ws + p.b * q.ws_one;
    int bi, bj;
    sym_tile(p.t, bi, bj);
    const float* in = (const float*)(ws + w_sym(q.sp, q.Lp, SYMS)) + (long long)p.t * q.splits * (T * T);
    float* C = (float*)lds;
    for (int e = (int)threadIdx.x; e < T * T; e += WG) {
        float v = in[e];
        for (int k = 1; k < q.splits; ++k) v += in[(long long)k * (T * T) + e];
        C[e / T * CP<T> + e % T] = v;
    }
    const float f = first ? norm_factor(q, ws, eps, s4) : 1.0f;
    __syncthreads();
    store_sym<T>(C, ws + w_sym(q.sp, q.Lp, 0), nullptr, q.sp, bi, bj, alpha * f * f, 0.0f, 0.0f);
}

// One or two products of symmetric matrices (numbers of the workspace's):
// c = alpha a b + beta d + gamma I.
struct SymJob {
    int a, b, c, d;
    float alpha, beta, gamma;
};
template <int T>
__global__ __launch_bounds__(WG, 2) void k_orth_sym(Table tb, SymJob j0, SymJob j1) {
    extern __shared__ __align__(16) unsigned char lds[];
    const Place p = place(tb, [](const OMat& q) { return sym_tiles<T>(q); });
    const OMat& q = tb.mat[p.mat];
    const SymJob& j = blockIdx.y ? j1 : j0;
    char* ws = q.ws + p.b * q.ws_one;
    int bi, bj;
    sym_tile(p.t, bi, bj);
    const long long pitch = (long long)q.sp * 4;
    auto sym = [&](int i) { return ws + w_sym(q.sp, q.Lp, i); };
    product_tile<T, 2, 2>(sym(j.a) + bi * T * pitch, pitch, sym(j.b) + bj * T * pitch, pitch, 0, q.sp / 32, lds);
    store_sym<T>((float*)lds, sym(j.c), j.d < 0 ? nullptr : sym(j.d), q.sp, bi, bj, j.alpha, j.beta, j.gamma);
}

// Q X: the next block's X and its transpose, or the result.
template <int T, int NP, typename TO, bool LAST>
__global__ __launch_bounds__(WG, 2) void k_orth_apply(Table tb, int Q, int xt, float alpha, float eps, int first) {
    extern __shared__ __align__(16) unsigned char lds[];
    __shared__ float s4[WG / 64];
    const Place p = place(tb, [](const OMat& q) { return (q.sp / T) * (q.Lp / T); });
    const OMat& q = tb.mat[p.mat];
    char* ws = q.ws + p.b * q.ws_one;
    const int ts = q.sp / T, i = p.t % ts, k = p.t / ts;  // tiles of one row of Xt are neighbours
    const char* qm = ws + w_sym(q.sp, q.Lp, Q) + (long long)i * T * q.sp * 4;
    const char* xm = ws + w_xt(q.sp, q.Lp, xt) + (long long)k * T * q.sp * (2 * NP);
    const bool tall = LAST && q.m > q.n;  // then the tile's rows are those of Xt
    if (tall) product_tile<T, NP, 2>(xm, (long long)q.sp * (2 * NP), qm, (long long)q.sp * 4, 0, q.sp / 32, lds);
    else product_tile<T, 2, NP>(qm, (long long)q.sp * 4, xm, (long long)q.sp * (2 * NP), 0, q.sp / 32, lds);
    float* C = (float*)lds;
    const float f = alpha * (first ? norm_factor(q, ws, eps, s4) : 1.0f);
    if constexpr (LAST) {
        TO* o = (TO*)q.o + p.b * q.bstride_o;
        const int r0 = (tall ? k : i) * T, c0 = (tall ? i : k) * T;
        for (int e = (int)threadIdx.x; e < T * T; e += WG) {
            const int r = r0 + e / T, c = c0 + e % T;
            if (r < q.m && c < q.n) o[r * q.ld_o + c] = from_f32<TO>(f * C[e / T * CP<T> + e % T]);
        }
    } else {
        for (int e = (int)threadIdx.x; e < T * T; e += WG) C[e / T * CP<T> + e % T] *= f;
        __syncthreads();
        store_tile<T, 2>(C, ws + W_X, q.Lp, i * T, k * T, false);
        store_tile<T, 2>(C, ws + w_xt(q.sp, q.Lp, xt ^ 1), q.sp, k * T, i * T, true);
    }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
struct Group {
    Table tb;
    int entry[OM], first[OM];  // of the list, and the first matrix of its batch
    int tile;
    size_t bytes;
};

long long up(long long n, long long k) { return (n + k - 1) / k * k; }

// The list cut into groups that share their launches and, one after the other,
// the workspace.  A group ends when its matrices alone fill the chip several
// times over, so that a long list or batch takes no more workspace than that.
std::vector<Group> groups_of(const OrthMat* mats, int count) {
    std::vector<Group> v;
    auto tiles = [](int s, int T) { const long long t = (s + T - 1) / T; return t * (t + 1) / 2; };
    int i = 0, b = 0;  // the next matrix
    while (i < count) {
        Group g{};
        long long work = 0;
        int n = 0, many[OM];
        while (i < count && n < OM && work < 2048) {
            const int s = std::min(mats[i].m, mats[i].n), L = std::max(mats[i].m, mats[i].n);
            const long long one = tiles(s, 128) + (up(s, 128) * up(L, 128) >> 20);
            const int take = (int)std::min<long long>(mats[i].batch - b, std::max(1LL, (2048 - work + one - 1) / one));
            g.first[n] = b;
            g.entry[n] = i;
            many[n++] = take;
            work += one * take;
            b += take;
            if (b == mats[i].batch) {
                ++i;
                b = 0;
            }
        }
        g.tile = work >= 256 ? 128 : 64;
        long long cells = 0;
        for (int k = 0; k < n; ++k) cells += tiles(std::min(mats[g.entry[k]].m, mats[g.entry[k]].n), g.tile) * many[k];
        for (int k = 0; k < n; ++k) {
            const OrthMat& q = mats[g.entry[k]];
            OMat& o = g.tb.mat[k];
            o.ld = q.ld;
            o.ld_o = q.ld_o;
            o.bstride = q.bstride;
            o.bstride_o = q.bstride_o;
            o.batch = many[k];
            o.m = q.m;
            o.n = q.n;
            o.s = std::min(q.m, q.n);
            o.L = std::max(q.m, q.n);
            o.sp = (int)up(o.s, g.tile);
            o.Lp = (int)up(o.L, g.tile);
            // parts over L until there are two workgroups a CU, each of 8 steps at least
            o.splits = (int)std::max(1LL, std::min<long long>(512 / std::max(1LL, cells), o.Lp / 256));
            o.ws_one = up(w_sym(o.sp, o.Lp, SYMS) +
                              (o.splits > 1 ? tiles(o.s, g.tile) * o.splits * g.tile * g.tile * 4 : 0), 256);
            g.bytes += (size_t)(o.ws_one * o.batch);
        }
        g.tb.count = n;
        v.push_back(g);
    }
    return v;
}

template <typename F>
unsigned number(Table& tb, F per) {
    long long n = 0;
    for (int i = 0; i < tb.count; ++i) {
        tb.start[i] = (int)n;
        n += (long long)per(tb.mat[i]) * tb.mat[i].batch;
    }
    for (int i = tb.count; i <= OM; ++i) tb.start[i] = (int)n;
    return (unsigned)n;
}

// What bounds a step: p on [0, lambda] (|p| <= p) and the next lambda.
struct Bound {
    double p, lambda;
};
Bound bound_of(const double* c, double lambda) {
    auto p = [&](double y) { return c[0] + y * (c[1] + y * c[2]); };
    Bound b{std::max(fabs(p(0.0)), fabs(p(lambda))), lambda * p(lambda) * p(lambda)};
    auto at = [&](double y, bool vertex) {
        if (!(y > 0.0 && y < lambda)) return;
        if (vertex) b.p = std::max(b.p, fabs(p(y)));
        b.lambda = std::max(b.lambda, y * p(y) * p(y));
    };
    if (c[2] != 0.0) at(-c[1] / (2.0 * c[2]), true);
    // x p(x^2) has its extremes where 5 c y^2 + 3 b y + a = 0
    const double d = 9.0 * c[1] * c[1] - 20.0 * c[2] * c[0];
    if (c[2] != 0.0 && d >= 0.0) {
        at((-3.0 * c[1] - sqrt(d)) / (10.0 * c[2]), false);
        at((-3.0 * c[1] + sqrt(d)) / (10.0 * c[2]), false);
    } else if (c[2] == 0.0 && c[1] != 0.0) {
        at(-c[0] / (3.0 * c[1]), false);
    }
    b.p = std::min(std::max(b.p, 1e-30), 1e30);
    b.lambda = std::min(std::max(b.lambda, 1e-30), 1e30);
    return b;
}
// The exponent e with bound * 2^e in (2^13, 2^14] (fp16 ends at 2^16).
int exponent(double bound) {
    int e;
    frexp(bound * 1.01, &e);
    return 14 - e;
}
float pow2(int e) { return (float)ldexp(1.0, std::max(-140, std::min(120, e))); }

template <typename T, int TILE>
hipError_t orth_group(Group& g, int steps, const double* coef, double eps_, hipStream_t st) {
    constexpr int NP = sizeof(T) == 4 ? 2 : 1;
    // (see the head of this file)
    constexpr double MAX_GROWTH = std::is_same<T, bf16>::value ? 2.1e4 : std::is_same<T, f16>::value ? 150.0 : 12.5;
    const float eps = (float)eps_;
    Table& tb = g.tb;
    hipError_t err = hipSuccess;
    auto run = [&](auto kernel, unsigned grid, unsigned grid_y, int lds, auto... args) {
        if (err != hipSuccess || grid == 0) return;
        if (lds && (err = ensure_dyn_lds((const void*)kernel, lds)) != hipSuccess) return;
        hipLaunchKernelGGL(kernel, dim3(grid, grid_y), dim3(WG), lds, st, tb, args...);
        err = hipGetLastError();
    };
    auto syms = [](const OMat& q) { const int t = q.sp / TILE; return t * (t + 1) / 2; };
    run(k_orth_amax<T>, number(tb, [](const OMat& q) { return std::min<long long>(MAXA, ((long long)q.m * q.n + 16383) / 16384); }), 1, 0);
    run(k_orth_prep<T>, number(tb, [](const OMat& q) { return std::min<long long>(MAXP, (long long)(q.sp / 64) * (q.Lp / 64)); }), 1, 0);
    double lambda = 1.0;
    int xt = 0, ex = 0, step = 0;  // X is stored times 2^ex (and norm_factor in the first block)
    constexpr int lds22 = product_lds<TILE, 2, 2>();
    for (bool first = true; step < steps; first = false) {
        int len = 0;
        double growth = 1.0, l = lambda;
        while (step + len < steps) {
            if (len && growth > MAX_GROWTH) break;
            const Bound b = bound_of(coef + 3 * (step + len), l);
            growth *= b.p * b.p;
            l = b.lambda;
            ++len;
        }
        const bool last = step + len == steps;
        int ea = exponent(lambda);
        const float galpha = pow2(ea - 2 * ex);
        const unsigned gram = number(tb, [&](const OMat& q) { return syms(q) * q.splits; });
        if (first && NP == 1) run(k_orth_gram<TILE, 1>, gram, 1, product_lds<TILE, 1, 1>(), galpha, eps, 1);
        else run(k_orth_gram<TILE, 2>, gram, 1, lds22, galpha, eps, (int)first);
        run(k_orth_parts<TILE>, number(tb, [&](const OMat& q) { return q.splits > 1 ? syms(q) : 0; }), 1,
            TILE * CP<TILE> * 4, galpha, eps, (int)first);
        const unsigned sym = number(tb, syms);
        int Q = -1, eq = 0;
        double qb = 1.0;
        for (int k = 0; k < len; ++k, ++step) {
            const double* c = coef + 3 * step;
            const Bound b = bound_of(c, lambda);
            const int ep = exponent(b.p), et = exponent(b.p * lambda), en = exponent(b.lambda);
            int P = 2;
            while (P == Q) ++P;
            const SymJob jp{0, 0, P, 0, (float)(c[2] * pow2(ep - 2 * ea)), (float)(c[1] * pow2(ep - ea)), (float)(c[0] * pow2(ep))};
            run(k_orth_sym<TILE>, sym, 1, lds22, jp, jp);
            qb = std::min(qb * b.p, 1e30);
            const int eq2 = exponent(qb);
            int Q2 = P;
            if (Q >= 0) Q2 = 2 + 3 - (Q - 2) - (P - 2);
            const SymJob jq{P, Q, Q2, -1, pow2(eq2 - ep - eq), 0.0f, 0.0f};
            const SymJob jt{P, 0, 1, -1, pow2(et - ep - ea), 0.0f, 0.0f};
            if (k + 1 < len) {
                if (Q >= 0) run(k_orth_sym<TILE>, sym, 2, lds22, jt, jq);
                else run(k_orth_sym<TILE>, sym, 1, lds22, jt, jt);
                const SymJob ja{1, P, 0, -1, pow2(en - et - ep), 0.0f, 0.0f};
                run(k_orth_sym<TILE>, sym, 1, lds22, ja, ja);
            } else if (Q >= 0) {
                run(k_orth_sym<TILE>, sym, 1, lds22, jq, jq);
            }
            eq = Q >= 0 ? eq2 : ep;
            Q = Q2;
            ea = en;
            lambda = b.lambda;
        }
        const unsigned app = number(tb, [](const OMat& q) { return (q.sp / TILE) * (q.Lp / TILE); });
        const int ex2 = exponent(sqrt(lambda));
        constexpr int lds_a = product_lds<TILE, 2, NP>();
        const float a = pow2((last ? 0 : ex2) - eq - ex);
        if (last) {
            if (first) run(k_orth_apply<TILE, NP, T, true>, app, 1, lds_a, Q, xt, a, eps, 1);
            else run(k_orth_apply<TILE, 2, T, true>, app, 1, lds22, Q, xt, a, eps, 0);
        } else {
            if (first) run(k_orth_apply<TILE, NP, T, false>, app, 1, lds_a, Q, xt, a, eps, 1);
            else run(k_orth_apply<TILE, 2, T, false>, app, 1, lds22, Q, xt, a, eps, 0);
            xt ^= 1;
        }
        ex = ex2;
    }
    return err;
}

template <typename T>
hipError_t orth_t(const OrthMat* mats, int count, int steps, const double* coef, double eps, Ws ws, hipStream_t st) {
    for (Group& g : groups_of(mats, count)) {
        char* at = (char*)ws.p;
        for (int k = 0; k < g.tb.count; ++k) {
            OMat& o = g.tb.mat[k];
            const OrthMat& q = mats[g.entry[k]];
            o.g = (const T*)q.g + g.first[k] * q.bstride;
            o.o = (T*)q.o + g.first[k] * q.bstride_o;
            o.ws = at;
            at += o.ws_one * o.batch;
        }
        const hipError_t e = g.tile == 128 ? orth_group<T, 128>(g, steps, coef, eps, st)
                                           : orth_group<T, 64>(g, steps, coef, eps, st);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

size_t orth_ws_bytes(int, const OrthMat* mats, int count) {
    size_t n = 0;
    for (const Group& g : groups_of(mats, count)) n = std::max(n, g.bytes);
    return n;
}

hipError_t launch_orth(int dtype, const OrthMat* mats, int count, int steps, const double* coef, double eps, Ws ws,
                       hipStream_t st) {
    if (dtype == 0) return orth_t<float>(mats, count, steps, coef, eps, ws, st);
    if (dtype == 1) return orth_t<f16>(mats, count, steps, coef, eps, ws, st);
    return orth_t<bf16>(mats, count, steps, coef, eps, ws, st);
}

}  // namespace sb
