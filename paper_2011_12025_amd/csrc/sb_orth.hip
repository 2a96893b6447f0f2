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
// steps of the default coefficients are blocks of 3 and 2 for 16-bit updates and of
// 2, 2 and 1 for fp32.  The
// error is then that of an fp32 iteration, before the result is rounded (4096 x
// 4096, where an fp32 iteration is off by what follows in brackets: Gaussian 3.4e-6
// in fp32 and 6.4e-6 else (4.8e-6), one direction alone 2.9e-4 and 2.4e-4 (5.2e-4)).
// One block of five steps is off by 2e-4 for the gradient of a filter, but by
// 1.6e-2 for one direction of 515 rows.  All s x s matrices and all
// X but the first are pairs of fp16 numbers hi + lo (22 bits and a sign) times
// a power of two known beforehand from the polynomial's bounds; a product of
// two is three MFMAs hi hi + hi lo + lo hi with fp32 sums.  (Single fp16 numbers
// are too few for 16-bit updates too: the slopes of later steps multiply their
// rounding, which adds 1e-3 to 2e-3 of the norm for spectra without large
// gaps, 8e-3 for four directions alike, and 0.1 with coefficients that are
// steeper.)  The first X is one fp16 number for 16-bit updates (fp16 as it is,
// bf16 times a power of two: values below 2^-38 of the largest are cut) and a
// pair for fp32.
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
    int parts, unit0;               // of X X^T: workgroups of a tile, and the number of the entry's first one
    int scaled;                     // whether X is the update times a power of two (else as it is)
    int vec;                        // whether rows of the update / of the result are 16-byte aligned (bits 0 / 1)
};
struct Table {
    OMat mat[OM];
    int start[OM + 1];
    int count;
};

// The workspace of one matrix, in bytes from its start.
constexpr int MAXP = 1024;  // workgroups that make X, each with its sum of squares
constexpr int MAXA = 1024;  // workgroups that look for the largest value
constexpr long long W_SUM = 4 * MAXA, W_X = W_SUM + 4 * MAXP;  // [0]: the largest values
__host__ __device__ inline long long w_x_bytes(int sp, int Lp) { return (long long)sp * Lp * 4; }
// X, of which a block needs no more than X X^T, and its transpose twice: a block's
// and the next one's
__host__ __device__ inline long long w_xt(int sp, int Lp, int i) { return W_X + (1 + i) * w_x_bytes(sp, Lp); }
__host__ __device__ inline long long w_sym(int sp, int Lp, int i) {
    return W_X + 3 * w_x_bytes(sp, Lp) + i * ((long long)sp * sp * 4);
}
constexpr int SYMS = 5;  // A, T and three that P and Q take in turn

struct Place {  // of a workgroup
    int mat, b, t;  // entry, matrix of its batch, tile
};
// Workgroups go to the eight XCDs in turn; of every entry an XCD gets a run of
// neighbouring tiles, which share panels, since each L2 fetches for itself what
// it reads.  (Of every entry and not of the launch: they take unequal time.)
__device__ __forceinline__ int xcd_run(int k, int n) {
    const int x = k & 7, q = n >> 3, r = n & 7;
    return x * q + min(x, r) + (k >> 3);
}
template <typename F>  // per_of: workgroups of one matrix of an entry
__device__ __forceinline__ Place place(const Table& tb, F per_of, int bid) {
    const int l = lane_id();
    const int i = __popcll(__ballot(l < tb.count && bid >= tb.start[min(l, OM)])) - 1;
    const int t = xcd_run(bid - tb.start[i], tb.start[i + 1] - tb.start[i]), per = per_of(tb.mat[i]);
    return Place{i, t / per, t % per};
}

__host__ __device__ inline int amax_wgs(const OMat& q) {
    const long long n = ((long long)q.m * q.n + 4095) / 4096;
    return n < MAXA ? (int)n : MAXA;
}
__host__ __device__ inline int prep_wgs(const OMat& q) {
    const long long n = (long long)(q.sp / 64) * (q.Lp / 64);
    return n < MAXP ? (int)n : MAXP;
}

// ---------------------------------------------------------------------------
// Storage of a matrix (S), rows of one of
//   ONES   [k], single numbers
//   PAIRS  [k / 32][32 hi | 32 lo]
// so that a product's step reads whole lines of 128 bytes.  The value is the count
// of numbers of an element.
// ---------------------------------------------------------------------------
enum { ONES = 1, PAIRS = 2 };
constexpr int LO_AT = 64;  // bytes from hi to lo
template <int S>
__device__ __forceinline__ long long at_k(long long k) {  // bytes, k a multiple of 8
    return S == ONES ? k * 2 : (k >> 5) * 128 + (k & 31) * 2;
}

template <int S>
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
    char* p = row + at_k<S>(k);
    vstore<f16, 8>((f16*)p, hi);
    if (S == PAIRS) vstore<f16, 8>((f16*)(p + LO_AT), lo);
}

// An R x T piece in LDS (fp32, rows CP<T> apart) to rows r0.. and columns c0.. of a
// matrix with K columns; TURNED: its transpose.
template <int T> constexpr int CP = T + 1;

// Threads of a workgroup with tiles of side T: one wave a SIMD stands still for its
// own instructions and LDS reads where tiles of 64 are a CU's only one, so those
// have two, each with half of a stage's K (s = 512: 12.4 -> 11.0 us a product).
template <int T> constexpr int NT = T == 64 ? 512 : 256;

template <int T, int S, bool TURNED, int R = T, int THREADS = NT<T>>
__device__ __forceinline__ void store_tile(const float* C, char* dst, long long K, int r0, int c0) {
    constexpr int W = (TURNED ? R : T) / 8;  // eights of a stored row
    for (int e = (int)threadIdx.x; e < R * T / 8; e += THREADS) {
        const int r = e / W, k = (e % W) * 8;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = TURNED ? C[(k + i) * CP<T> + r] : C[r * CP<T> + k + i];
        store8<S>(dst + (long long)(r0 + r) * K * (2 * S), c0 + k, v);
    }
}

// ---------------------------------------------------------------------------
// The first X.
// ---------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(WG) void k_orth_amax(Table tb) {
    constexpr int V = 16 / (int)sizeof(T);
    __shared__ float s[WG / 64];
    const Place p = place(tb, [](const OMat& q) { return amax_wgs(q); }, (int)blockIdx.x);
    const OMat& q = tb.mat[p.mat];
    const T* g = (const T*)q.g + p.b * q.bstride;
    const int tid = (int)threadIdx.x, l = lane_id(), wgs = amax_wgs(q);
    float m = 0.0f;
    // rows of vectors, or one row of all where nothing lies between them
    const bool flat = q.ld == q.n;
    const long long cols = flat ? (long long)q.m * q.n : q.n, rows = flat ? 1 : q.m;
    const bool vec = q.vec & 1;
    const int step = vec ? V : 1;
    const long long across = (cols + step - 1) / step, count = rows * across, all = (long long)wgs * WG;
#pragma unroll 4
    for (long long x = (long long)p.t * WG + tid; x < count; x += all) {
        const long long r = flat ? 0 : x / across, c = (x - r * across) * step;
        const T* from = g + r * q.ld + c;
        if (vec && c + V <= cols) {
            Vec<T, V> y;
            y.raw = *reinterpret_cast<const uint4*>(from);
#pragma unroll
            for (int k = 0; k < V; ++k) m = fmaxf(m, fabsf(to_f32(y.e[k])));
        } else {
            for (int k = 0; k < step; ++k)
                if (c + k < cols) m = fmaxf(m, fabsf(to_f32(from[k])));
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
    if (l == 0) s[tid >> 6] = m;
    __syncthreads();
    if (tid == 0) ((float*)(q.ws + p.b * q.ws_one))[p.t] = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
}

// The sum of n floats (fixed order) or their maximum, over a workgroup.  The same
// value whatever its size: lane t of a wave takes every 64th, all waves alike.
template <bool MAX>
__device__ __forceinline__ float wave_reduce(const float* p, int n) {
    float v = 0.0f;
#pragma unroll 8
    for (int i = lane_id(); i < n; i += 64) v = MAX ? fmaxf(v, p[i]) : v + p[i];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const float w = __shfl_xor(v, o, 64);
        v = MAX ? fmaxf(v, w) : v + w;
    }
    return v;
}

// The power of two that brings the largest value to [2^13, 2^14).  An fp16 update
// is taken as it is: its squares and their sums keep
// within fp32, and MFMA reads fp16 subnormals.
__device__ __forceinline__ int scale_of(const OMat& q, const char* ws) {
    if (!q.scaled) return 0;
    const float m = wave_reduce<true>((const float*)ws, amax_wgs(q));
    int e = 0;
    if (m > 0.0f && m < INFINITY) frexpf(m, &e);
    return max(-126, min(126, m > 0.0f ? 14 - e : 0));
}

// 1 / (|G| + eps) for X as it is stored: 0 for zeros, NaN where |G| is not finite.
__device__ __forceinline__ float norm_factor(const OMat& q, const char* ws, float eps) {
    const int e = scale_of(q, ws);
    const float t = wave_reduce<false>((const float*)(ws + W_SUM), prep_wgs(q));
    return t == 0.0f ? 0.0f : t < INFINITY ? 1.0f / (sqrtf(t) + ldexpf(eps, e)) : NAN;
}

// X [sp][Lp] and its transpose [Lp][sp] from the update, and its squares.
template <typename T>
__global__ __launch_bounds__(WG) void k_orth_prep(Table tb) {
    constexpr int S = sizeof(T) == 4 ? PAIRS : ONES, V = 16 / (int)sizeof(T);
    __shared__ float C[64 * CP<64>];
    __shared__ float s4[WG / 64];
    const Place p = place(tb, [](const OMat& q) { return prep_wgs(q); }, (int)blockIdx.x);
    const OMat& q = tb.mat[p.mat];
    const T* g = (const T*)q.g + p.b * q.bstride;
    char* ws = q.ws + p.b * q.ws_one;
    const int e = scale_of(q, ws), tid = (int)threadIdx.x;
    const bool tall = q.m > q.n;
    const int mp = tall ? q.Lp : q.sp, np = tall ? q.sp : q.Lp, tn = np / 64, tiles = (mp / 64) * tn, wgs = prep_wgs(q);
    char* X = ws + W_X;                     // [sp][Lp]
    char* Xt = ws + w_xt(q.sp, q.Lp, 0);    // [Lp][sp]
    float sum = 0.0f;
    for (int t = p.t; t < tiles; t += wgs) {
        const int r0 = t / tn * 64, c0 = t % tn * 64;
        if (q.vec & 1) {
#pragma unroll
            for (int i = 0; i < 64 * 64 / V / WG; ++i) {
                const int x = i * WG + tid, r = x / (64 / V), c = x % (64 / V) * V;
                Vec<T, V> in;
                in.raw = uint4{0u, 0u, 0u, 0u};
                const T* row = g + (r0 + r) * q.ld + c0;
                if (r0 + r < q.m && c0 + c + V <= q.n) in.raw = *reinterpret_cast<const uint4*>(row + c);
                else if (r0 + r < q.m)
                    for (int k = 0; k < V; ++k)
                        if (c0 + c + k < q.n) in.e[k] = row[c + k];
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    const float v = ldexpf(to_f32(in.e[k]), e);
                    C[r * CP<64> + c + k] = v;
                    sum += v * v;
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int r = i * 4 + (tid >> 6), c = tid & 63;
                const float v = r0 + r < q.m && c0 + c < q.n ? ldexpf(to_f32(g[(r0 + r) * q.ld + c0 + c]), e) : 0.0f;
                C[r * CP<64> + c] = v;
                sum += v * v;
            }
        }
        __syncthreads();
        store_tile<64, S, false, 64, WG>(C, tall ? Xt : X, np, r0, c0);
        store_tile<64, S, true, 64, WG>(C, tall ? X : Xt, mp, c0, r0);
        __syncthreads();
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
    if (lane_id() == 0) s4[tid >> 6] = sum;
    __syncthreads();
    if (tid == 0) ((float*)(ws + W_SUM))[p.t] = (s4[0] + s4[1]) + (s4[2] + s4[3]);
}

// ---------------------------------------------------------------------------
// A T x T tile of A B^T, K in steps of 32 (of 64 where both operands are single
// numbers): both operands' rows go to LDS by DMA (16 bytes a lane) while the steps
// before are multiplied.  128 (64) bytes a row and step, its 16-byte chunks XORed by
// the pair (four) of rows, so that 16 rows lie in distinct ones of the 64 banks
// (XORed by the row, with 8 distinct, a read took twice the cycles).  Four waves,
// each a quarter of the tile in v_mfma_f32_32x32x16_f16.
// ---------------------------------------------------------------------------
template <int T> constexpr int MF = T / 64;  // 32 x 32 fragments of a wave, each way

template <int BYTES_ROW>
__device__ __forceinline__ int chunk_of(int row, int c) {  // where chunk c of a row lies
    return BYTES_ROW == 128 ? c ^ ((row >> 1) & 7) : c ^ ((row >> 2) & 3);
}

// Steps of 32 that a stage holds, and the elements of K of one: with tiles of 64 the
// latency of a stage (LDS reads, then the chain of MFMAs) counts, so it is longer.
// Products of single numbers take 64 elements in either.
template <int T> constexpr int KS = T == 64 ? 2 : 1;
template <int T, int NA, int NB> constexpr int STEP_K = NA + NB == 2 ? 64 : 32 * KS<T>;
template <int T, int NA, int NB> constexpr int stage_bytes() { return T * 2 * STEP_K<T, NA, NB> * (NA + NB); }
// Stages in LDS.  Tiles of 128: as many as leave room for two workgroups on a CU.
// Tiles of 64 are for products that do not fill the chip: one workgroup a CU,
// and what it has in flight against the latency of another XCD's results decides.
template <int T, int NA, int NB> constexpr int stages() {
    return T == 128 ? std::max(2, 66 * 1024 / stage_bytes<T, NA, NB>()) : 4;
}
template <int T, int NA, int NB> constexpr int product_lds() {
    return std::max(stages<T, NA, NB>() * stage_bytes<T, NA, NB>(), T * CP<T> * 4);
}

// All waves' DMA but the last `left` instructions of each has landed, and their
// reads of the stage before are done.
template <int LEFT>
__device__ __forceinline__ void product_barrier() {
    static_assert(LEFT < 64, "vmcnt");
    __builtin_amdgcn_s_waitcnt((LEFT & 15) | 7 << 4 | (LEFT >> 4) << 14);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

__device__ __forceinline__ floatx16 mfma(halfx8 a, halfx8 b, floatx16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

// 16 bytes a lane to the wave's 1 KB at `to`.
__device__ __forceinline__ void dma16(const char* from, unsigned char* to) {
    __builtin_amdgcn_global_load_lds(from, (lds_ptr)to, 16, 0, 0);
}

// rows of A and B from their first element on; the tile ends in LDS as fp32.  NA,
// NB: how they are stored.
//
// A wave's DMA instructions are spread over its MFMAs: a CU takes one (1 KB) in
// about 28 cycles, and a wave that issues a stage's eight in a row stands still
// until the last is taken.  Half of 4096 x 4096 x 4096 in three products: DMA alone
// 100 us, MFMAs with their LDS reads alone 112, together 207 and spread 196 (1.08
// PFLOP/s of MFMA, where a large library product reaches 1.21).  More stages (one
// workgroup of eight waves a CU), or operands read a stage ahead, were no faster.
// Of single numbers it takes 84 us (0.82 PFLOP/s, DMA and MFMAs in turn), and in steps
// of 32, whose instructions touch twice the lines for half of each, 106.
template <int T, int NA, int NB>
__device__ __forceinline__ void product_tile(const char* A, long long pa, const char* B, long long pb, int step0,
                                             int steps, unsigned char* lds) {
    constexpr bool ONE = NA + NB == 2;
    constexpr int RA = ONE ? 128 : 64 * NA, RB = ONE ? 128 : 64 * NB;  // bytes of a row and step
    constexpr int STAGE = stage_bytes<T, NA, NB>(), OB = T * RA, STEP = T * (RA + RB), NST = stages<T, NA, NB>();
    // Two groups of four waves take steps of 32 in turn, or halves of one step of 64.
    constexpr int GROUPS = NT<T> / WG, LOADERS = ONE ? NT<T> : WG, STEPS = ONE ? 1 : KS<T>;
    // DMA instructions of a thread and step; of a thread and stage
    constexpr int LA = T * RA / 16 / LOADERS, LB = T * RB / 16 / LOADERS, LH = LA + LB;
    constexpr int LOADS = ONE ? LH : STEPS * LH / GROUPS;
    static_assert(ONE || STEPS % GROUPS == 0, "a group takes whole steps of 32");
    // the three products of a 64 x 64 tile's one fragment in sums of their own:
    // an MFMA waits for the one before it on the same sum
    constexpr int CH = T == 64 ? NA + NB - 1 : 1;
    const int tid = (int)threadIdx.x & (LOADERS - 1), l = lane_id();
    const int wave = __builtin_amdgcn_readfirstlane(((int)threadIdx.x & (WG - 1)) >> 6);
    const int loader = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int group = GROUPS == 1 ? 0 : __builtin_amdgcn_readfirstlane((int)threadIdx.x / WG);
    const int ra = (wave >> 1) * (T / 2) + (l & 31), rb = (wave & 1) * (T / 2) + (l & 31);
    // this lane's 16 bytes of every instruction, from the operand's first row
    unsigned from[LH];
#pragma unroll
    for (int i = 0; i < LH; ++i) {
        const int chunks = (i < LA ? RA : RB) / 16, c = (i < LA ? i : i - LA) * LOADERS + tid, r = c / chunks;
        const int chunk = i < LA ? chunk_of<RA>(r, c % chunks) : chunk_of<RB>(r, c % chunks);
        from[i] = (unsigned)(r * (i < LA ? pa : pb) + chunk * 16);
    }
    auto dma = [&](int i, int s, int buf) {  // instruction i of stage s
        const int k = ONE ? 0 : i / LH * GROUPS + group, j = i % LH;
        const char* base = (j < LA ? A : B) + ((long long)(step0 + s) * STEPS + k) * (j < LA ? RA : RB);
        unsigned char* to = lds + buf * STAGE + k * STEP + (j < LA ? j : j - LA) * (LOADERS * 16) + (j < LA ? 0 : OB) +
                            loader * 1024;
        dma16(base + from[j], to);
    };
    floatx16 acc[CH][MF<T>][MF<T>] = {};
    for (int s = 0; s < min(NST - 1, steps); ++s)
#pragma unroll
        for (int i = 0; i < LOADS; ++i) dma(i, s, s);
    int at = 0;
    for (int s = 0; s < steps; ++s) {
        if (s + NST - 2 < steps) product_barrier<(NST - 2) * LOADS>();
        else product_barrier<0>();
        const unsigned char* cur = lds + at * STAGE;
        const bool more = s + NST - 1 < steps;
        const int into = at == 0 ? NST - 1 : at - 1;
        at = at + 1 == NST ? 0 : at + 1;
        constexpr int J = STEP_K<T, NA, NB> / 16 / GROUPS;
        halfx8 fa[J][NA][MF<T>], fb[J][NB][MF<T>];  // of the whole stage: their reads are in flight together
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int c = (ONE ? 2 * (J * group + j) : 2 * (j & 1)) + (l >> 5);
            const unsigned char* step = cur + (ONE ? 0 : ((j >> 1) * GROUPS + group) * STEP);
#pragma unroll
            for (int i = 0; i < MF<T>; ++i) {
#pragma unroll
                for (int h = 0; h < NA; ++h)
                    fa[j][h][i] = *(const halfx8*)(step + (ra + 32 * i) * RA + chunk_of<RA>(ra + 32 * i, 4 * h + c) * 16);
#pragma unroll
                for (int h = 0; h < NB; ++h)
                    fb[j][h][i] = *(const halfx8*)(step + OB + (rb + 32 * i) * RB +
                                                   chunk_of<RB>(rb + 32 * i, 4 * h + c) * 16);
            }
        }
        constexpr int MM = J * (NA + NB - 1) * MF<T> * MF<T>;  // MFMAs of a stage
        int m = 0, d = 0;
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int h = 0; h < NA + NB - 1; ++h) {  // hi hi, hi lo, lo hi
                constexpr int LO_A = NB == 2 ? 2 : 1;
                const int ha = NA == 2 && h == LO_A ? 1 : 0, hb = NB == 2 && h == 1 ? 1 : 0;
#pragma unroll
                for (int x = 0; x < MF<T>; ++x)
#pragma unroll
                    for (int y = 0; y < MF<T>; ++y) {
                        acc[h % CH][x][y] = mfma(fa[j][ha][x], fb[j][hb][y], acc[h % CH][x][y]);
                        ++m;
                        while (d * MM < m * LOADS) {
                            __builtin_amdgcn_sched_barrier(0);
                            if (more) dma(d, s + NST - 1, into);
                            __builtin_amdgcn_sched_barrier(0);
                            ++d;
                        }
                    }
            }
    }
#pragma unroll
    for (int h = 1; h < CH; ++h) acc[0][0][0] += acc[h][0][0];
    float* C = (float*)lds;
#pragma unroll
    for (int g = GROUPS - 1; g >= 0; --g) {  // the last group's sums, then the first's on top
        __syncthreads();
        if (g == group)
#pragma unroll
            for (int x = 0; x < MF<T>; ++x)
#pragma unroll
                for (int y = 0; y < MF<T>; ++y)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int i = (wave >> 1) * (T / 2) + 32 * x + (r & 3) + 8 * (r >> 2) + 4 * (l >> 5);
                        const int j = (wave & 1) * (T / 2) + 32 * y + (l & 31);
                        float& c = C[i * CP<T> + j];
                        c = g == GROUPS - 1 ? acc[0][x][y][r] : c + acc[0][x][y][r];
                    }
    }
    __syncthreads();
}

template <int T>
__device__ __forceinline__ int sym_tiles(const OMat& q) {
    const int t = q.sp / T;
    return t * (t + 1) / 2;
}
__device__ __forceinline__ void triangle(int t, int& i, int& j) {  // the t-th of (0, 0), (1, 0), (1, 1), ...
    i = (int)((sqrtf(8.0f * t + 1.0f) - 1.0f) * 0.5f);
    while ((i + 1) * (i + 2) / 2 <= t) ++i;
    while (i * (i + 1) / 2 > t) --i;
    j = t - i * (i + 1) / 2;
}
// The t-th tile with bi >= bj of n x n: strips of eight rows of tiles, each column
// by column, so that 64 neighbours (what an XCD works on at a time) read 16
// panels and not 35.
__device__ __forceinline__ void sym_tile(int t, int n, int& bi, int& bj) {
    int S = (int)((sqrtf(16.0f + 128.0f * t) - 4.0f) * (1.0f / 64.0f));  // 32 S^2 + 4 S tiles before strip S
    while (32 * (S + 1) * (S + 1) + 4 * (S + 1) <= t) ++S;
    while (32 * S * S + 4 * S > t) --S;
    const int local = t - 32 * S * S - 4 * S, h = min(8, n - 8 * S), square = 8 * S * h;
    if (local < square) {
        bj = local / h;
        bi = 8 * S + (local - bj * h);
    } else {
        triangle(local - square, bi, bj);
        bi += 8 * S;
        bj += 8 * S;
    }
}

// out = alpha C + beta D + gamma I for R x T cells at (r0, c0) of symmetric
// matrices [sp][sp], and their mirror image.
template <int T, int R>
__device__ __forceinline__ void store_sym(float* C, char* out, const char* D, int sp, int r0, int c0, bool mirror,
                                          float alpha, float beta, float gamma) {
    for (int e = (int)threadIdx.x; e < R * T / 8; e += NT<T>) {
        const int r = e / (T / 8), k = (e % (T / 8)) * 8, K = c0 + k;
        const long long row = (long long)(r0 + r) * sp * 4;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = alpha * C[r * CP<T> + k + i];
        if (D) {
            const Vec<f16, 8> hi = vload<f16, 8>((const f16*)(D + row + at_k<PAIRS>(K)));
            const Vec<f16, 8> lo = vload<f16, 8>((const f16*)(D + row + at_k<PAIRS>(K) + LO_AT));
#pragma unroll
            for (int i = 0; i < 8; ++i)
                v[i] += beta * ((float)hi.e[i] + (float)lo.e[i]) + (r0 + r == K + i ? gamma : 0.0f);
        }
        store8<PAIRS>(out + row, K, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) C[r * CP<T> + k + i] = v[i];
    }
    if (!mirror) return;
    __syncthreads();
    store_tile<T, PAIRS, true, R>(C, out, sp, c0, r0);
}

// One or two products that give symmetric matrices (numbers of the
// workspace's): c = alpha a b + beta d + gamma I, or c = alpha f^2 X X^T with f the
// norm's factor in the first block.  A tile is a workgroup's, or it is split over
// K among several (units) that leave their sums for k_orth_join:
//   whole >= 0: the tiles of the entries, of the first product and then of the
//     second, are numbered through; those from `whole` on have `parts` units each;
//   whole < 0 (X X^T alone): every entry's tiles have `parts` of its own.
struct SymJob {
    int a, b, c, d;
    float alpha, beta, gamma;
};
struct SymLaunch {
    SymJob job[2];
    int tiles;  // of one product
    int whole, parts, first;
    int leave;  // sums of every tile, for k_orth_steps
    float eps;
    float* sums;  // [unit][T * T], units counted from the first split tile's (whole < 0: from the first of all)
};

struct SymUnit {
    Place p;
    int job, part, parts;
    long long unit;
};
template <int T>
__device__ __forceinline__ SymUnit sym_unit(const Table& tb, const SymLaunch& s, int bid) {
    auto tiles = [](const OMat& q) { return sym_tiles<T>(q); };
    if (s.whole < 0) {
        Place p = place(tb, [](const OMat& q) { return sym_tiles<T>(q) * q.parts; }, bid);
        const OMat& q = tb.mat[p.mat];
        const int u = p.t, n = sym_tiles<T>(q);
        p.t = u / q.parts;
        return SymUnit{p, 0, u % q.parts, q.parts, q.unit0 + ((long long)p.b * n + p.t) * q.parts + u % q.parts};
    }
    const int over = bid - s.whole, tile = over < 0 ? bid : s.whole + over / s.parts, job = tile >= s.tiles;
    return SymUnit{place(tb, tiles, tile - job * s.tiles), job, over < 0 ? 0 : over % s.parts, over < 0 ? 1 : s.parts, over};
}

// C: R rows of the tile from row `part` R on.
template <int T, int R, bool GRAM>
__device__ __forceinline__ void sym_out(const OMat& q, char* ws, const SymLaunch& s, const SymJob& j, int t, int part,
                                        float* C) {
    int bi, bj;
    sym_tile(t, q.sp / T, bi, bj);
    auto sym = [&](int i) { return ws + w_sym(q.sp, q.Lp, i); };
    float alpha = j.alpha;
    if (GRAM && s.first) {
        const float f = norm_factor(q, ws, s.eps);
        alpha *= f * f;
    }
    store_sym<T, R>(C, sym(j.c), GRAM || j.d < 0 ? nullptr : sym(j.d), q.sp, bi * T + part * R, bj * T, bi != bj,
                    alpha, j.beta, j.gamma);
}

template <int T, int S, bool GRAM>
__global__ __launch_bounds__(NT<T>, 2) void k_orth_sym(Table tb, SymLaunch s) {
    extern __shared__ __align__(16) unsigned char lds[];
    const SymUnit u = sym_unit<T>(tb, s, (int)blockIdx.x);
    const OMat& q = tb.mat[u.p.mat];
    const SymJob& j = s.job[u.job];
    char* ws = q.ws + u.p.b * q.ws_one;
    int bi, bj;
    sym_tile(u.p.t, q.sp / T, bi, bj);
    const int K = GRAM ? q.Lp : q.sp, steps = K / STEP_K<T, S, S>;
    const int k0 = (int)((long long)steps * u.part / u.parts), k1 = (int)((long long)steps * (u.part + 1) / u.parts);
    const long long pitch = (long long)K * (2 * S);
    const char* A = GRAM ? ws + W_X : ws + w_sym(q.sp, q.Lp, j.a);
    const char* B = GRAM ? A : ws + w_sym(q.sp, q.Lp, j.b);
    product_tile<T, S, S>(A + bi * T * pitch, pitch, B + bj * T * pitch, pitch, k0, k1 - k0, lds);
    float* C = (float*)lds;
    if (u.parts > 1 || s.leave) {
        float4* out = (float4*)(s.sums + u.unit * (T * T));
        for (int e = (int)threadIdx.x; e < T * T / 4; e += NT<T>) {
            const float* c = C + e / (T / 4) * CP<T> + e % (T / 4) * 4;
            out[e] = float4{c[0], c[1], c[2], c[3]};
        }
        return;
    }
    sym_out<T, T, GRAM>(q, ws, s, j, u.p.t, 0, C);
}

// The parts of the split tiles added in their order, a few rows a workgroup.
template <int T> constexpr int JOIN_ROWS = T == 64 ? 32 : 16;
template <int T, bool GRAM>
__global__ __launch_bounds__(NT<T>) void k_orth_join(Table tb, SymLaunch s) {
    constexpr int R = JOIN_ROWS<T>, N = R * T / 4 / NT<T>;  // vectors of a thread
    __shared__ float C[R * CP<T>];
    SymUnit u;
    int slice;
    if (s.whole < 0) {  // (the launch is numbered by slices of the tiles with several parts)
        u.p = place(tb, [](const OMat& q) { return q.parts > 1 ? sym_tiles<T>(q) * (T / R) : 0; }, (int)blockIdx.x);
        const OMat& q = tb.mat[u.p.mat];
        slice = u.p.t % (T / R);
        u.p.t /= T / R;
        u.job = 0;
        u.parts = q.parts;
        u.unit = q.unit0 + ((long long)u.p.b * sym_tiles<T>(q) + u.p.t) * q.parts;
    } else {
        slice = (int)blockIdx.x % (T / R);
        u = sym_unit<T>(tb, s, s.whole + (int)blockIdx.x / (T / R) * s.parts);
    }
    const OMat& q = tb.mat[u.p.mat];
    const float4* in = (const float4*)(s.sums + u.unit * (T * T) + slice * (R * T));
    float4 sum[N] = {};
#pragma unroll 4
    for (int k = 0; k < u.parts; ++k)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float4 v = in[(long long)k * (T * T / 4) + i * NT<T> + (int)threadIdx.x];
            sum[i] = float4{sum[i].x + v.x, sum[i].y + v.y, sum[i].z + v.z, sum[i].w + v.w};
        }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int e = i * NT<T> + (int)threadIdx.x;
        float* c = C + e / (T / 4) * CP<T> + e % (T / 4) * 4;
        c[0] = sum[i].x;
        c[1] = sum[i].y;
        c[2] = sum[i].z;
        c[3] = sum[i].w;
    }
    __syncthreads();
    sym_out<T, R, GRAM>(q, q.ws + u.p.b * q.ws_one, s, s.job[u.job], u.p.t, slice, C);
}

// A block of steps on matrices of one tile (s <= 64) without leaving a workgroup:
// from the sums of X X^T to Q, everything in LDS.  As launches of their own its
// products took 4.6 us each, whatever they compute (a filter of 64 x 576, 13
// products: 60 us; here the whole block takes 7.4 to 11 us).  Four waves a product,
// the eight share T and Q.
struct Steps {
    int len, first, Q;  // Q: where it goes
    float a0, eps;      // A = a0 f^2 X X^T
    const float* sums;
    struct One {
        float aa, a, i, t, n, q;  // P = aa A A + a A + i I,  T = t P A,  A = n T P,  Q = q P Q
    } one[8];  // (blocks are no longer)
};
constexpr int STEP_MAX = 8;
constexpr int STEPS_LDS = 5 * 64 * 256;

// Where 8 elements k.. of a row lie in a matrix in LDS (the hi part; lo is chunk + 4).
__device__ __forceinline__ int step_at(int row, int k, bool lo) {
    return (k >> 5) * (64 * 128) + row * 128 + chunk_of<128>(row, (k >> 3 & 3) + (lo ? 4 : 0)) * 16;
}

// c = alpha (a b^T)^T + beta d + gamma I by four waves (d nullptr: the product
// alone).  All of them are symmetric up to rounding, and the product is stored
// transposed, four elements a lane.  The order of the factors counts: with
// T = P A^T (a = A, b = P) the next A = P T^T = P A P^T is a congruence, which keeps
// it symmetric; as P P A^T the little by which P and A do not commute grows as
// an error of A does (bf16, 64 x 64, five steps in a block: 8e-3 off and not 1.7e-3,
// the rounding of the result).
__device__ __forceinline__ void step_product(const unsigned char* a, const unsigned char* b, unsigned char* c,
                                             const unsigned char* d, float alpha, float beta, float gamma) {
    const int l = lane_id(), wave = (int)threadIdx.x >> 6 & 3;
    const int ra = (wave >> 1) * 32 + (l & 31), rb = (wave & 1) * 32 + (l & 31);
    halfx8 fa[4][2], fb[4][2];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int k = 16 * j + 8 * (l >> 5);
            fa[j][h] = *(const halfx8*)(a + step_at(ra, k, h));
            fb[j][h] = *(const halfx8*)(b + step_at(rb, k, h));
        }
    floatx16 acc[3] = {};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        acc[0] = mfma(fa[j][0], fb[j][0], acc[0]);
        acc[1] = mfma(fa[j][0], fb[j][1], acc[1]);
        acc[2] = mfma(fa[j][1], fb[j][0], acc[2]);
    }
    acc[0] += acc[1] + acc[2];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int k = (wave >> 1) * 32 + 8 * q + 4 * (l >> 5), at = (k & 4) * 2;  // this lane's rows k..k+3 of column rb
        unsigned char* hi = c + step_at(rb, k & ~7, false) + at;
        unsigned char* lo = c + step_at(rb, k & ~7, true) + at;
        Vec<f16, 4> dh, dl, h, g;
        if (d) {
            dh = vload<f16, 4>((const f16*)(d + (hi - c)));
            dl = vload<f16, 4>((const f16*)(d + (lo - c)));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float v = alpha * acc[0][4 * q + i];
            if (d) v += beta * ((float)dh.e[i] + (float)dl.e[i]) + (rb == k + i ? gamma : 0.0f);
            asm("" : "+v"(v));  // (see store8)
            h.e[i] = (f16)v;
            g.e[i] = (f16)(v - (float)h.e[i]);
        }
        vstore<f16, 4>((f16*)hi, h);
        vstore<f16, 4>((f16*)lo, g);
    }
}

__global__ __launch_bounds__(512) void k_orth_steps(Table tb, Steps st) {
    extern __shared__ __align__(16) unsigned char lds[];
    const Place p = place(tb, [](const OMat&) { return 1; }, (int)blockIdx.x);
    const OMat& q = tb.mat[p.mat];
    char* ws = q.ws + p.b * q.ws_one;
    const int tid = (int)threadIdx.x, group = __builtin_amdgcn_readfirstlane(tid >> 8);
    auto sym = [&](int i) { return lds + i * (64 * 256); };
    const float f = st.first ? norm_factor(q, ws, st.eps) : 1.0f;
    {
        const int row = tid >> 3, k = (tid & 7) * 8;
        const float* in = st.sums + (q.unit0 + (long long)p.b * q.parts) * 4096 + row * 64 + k;
        float v[8] = {};
#pragma unroll 4
        for (int n = 0; n < q.parts; ++n) {
            const float4 x = *(const float4*)(in + n * 4096LL), y = *(const float4*)(in + n * 4096LL + 4);
            const float w[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += w[i];
        }
        Vec<f16, 8> hi, lo;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float x = v[i] * (st.a0 * f * f);
            asm("" : "+v"(x));  // (see store8)
            hi.e[i] = (f16)x;
            lo.e[i] = (f16)(x - (float)hi.e[i]);
        }
        vstore<f16, 8>((f16*)(sym(0) + step_at(row, k, false)), hi);
        vstore<f16, 8>((f16*)(sym(0) + step_at(row, k, true)), lo);
    }
    int Q = -1;
    for (int n = 0; n < st.len; ++n) {
        const Steps::One& o = st.one[n];
        const int P = Q == 2 ? 3 : 2, Q2 = Q < 0 ? P : 9 - Q - P;
        const bool more = n + 1 < st.len;
        __syncthreads();
        if (group == 0) step_product(sym(0), sym(0), sym(P), sym(0), o.aa, o.a, o.i);
        __syncthreads();
        if (group == 0 && more) step_product(sym(0), sym(P), sym(1), nullptr, o.t, 0.0f, 0.0f);
        if (group == 1 && Q >= 0) step_product(sym(Q), sym(P), sym(Q2), nullptr, o.q, 0.0f, 0.0f);
        if (more) {
            __syncthreads();
            if (group == 0) step_product(sym(1), sym(P), sym(0), nullptr, o.n, 0.0f, 0.0f);
        }
        Q = Q2;
    }
    __syncthreads();
    char* out = ws + w_sym(q.sp, q.Lp, st.Q);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int e = i * 512 + tid, row = e >> 4, c = e & 15;  // 16 bytes c of the row
        *(uint4*)(out + row * 256 + c * 16) = *(const uint4*)(sym(Q) + step_at(row, (c >> 3) * 32 + (c & 3) * 8, c & 4));
    }
}

// Q X: the next block's X and its transpose, or the result.  S: how X is stored.
struct Apply {
    int Q, xt, first;
    float alpha, eps;
};
template <int T, int S, typename TO, bool LAST>
__global__ __launch_bounds__(NT<T>, 2) void k_orth_apply(Table tb, Apply ap) {
    extern __shared__ __align__(16) unsigned char lds[];
    const Place p = place(tb, [](const OMat& q) { return (q.sp / T) * (q.Lp / T); }, (int)blockIdx.x);
    const OMat& q = tb.mat[p.mat];
    char* ws = q.ws + p.b * q.ws_one;
    // strips of eight rows of Q, each along L
    const int strip = p.t / (8 * (q.Lp / T)), h = min(8, q.sp / T - 8 * strip), local = p.t - strip * (8 * (q.Lp / T));
    const int k = local / h, i = 8 * strip + (local - k * h);
    const long long pq = (long long)q.sp * 4, px = (long long)q.sp * (2 * S);
    const char* qm = ws + w_sym(q.sp, q.Lp, ap.Q) + i * T * pq;
    const char* xm = ws + w_xt(q.sp, q.Lp, ap.xt) + k * T * px;
    const bool tall = LAST && q.m > q.n;  // then the tile's rows are those of the transpose
    const int steps = q.sp / STEP_K<T, PAIRS, S>;
    if (tall) product_tile<T, S, PAIRS>(xm, px, qm, pq, 0, steps, lds);
    else product_tile<T, PAIRS, S>(qm, pq, xm, px, 0, steps, lds);
    float* C = (float*)lds;
    const float alpha = (ap.first ? norm_factor(q, ws, ap.eps) : 1.0f) * ap.alpha;
    for (int e = (int)threadIdx.x; e < T * T / 8; e += NT<T>) {  // each thread its own eights
        float* v = C + e / (T / 8) * CP<T> + e % (T / 8) * 8;
#pragma unroll
        for (int x = 0; x < 8; ++x) v[x] *= alpha;
    }
    __syncthreads();
    if constexpr (LAST) {
        TO* o = (TO*)q.o + p.b * q.bstride_o;
        const int r0 = (tall ? k : i) * T, c0 = (tall ? i : k) * T;
        constexpr int V = 16 / (int)sizeof(TO);
        for (int e = (int)threadIdx.x; e < T * T / V; e += NT<T>) {
            const int x = e / (T / V), y = e % (T / V) * V, r = r0 + x, c = c0 + y;
            Vec<TO, V> v;
#pragma unroll
            for (int n = 0; n < V; ++n) v.e[n] = from_f32<TO>(C[x * CP<T> + y + n]);
            if (r >= q.m) continue;
            TO* to = o + r * q.ld_o + c;
            if ((q.vec & 2) && c + V <= q.n) *reinterpret_cast<uint4*>(to) = v.raw;
            else
                for (int n = 0; n < V; ++n)
                    if (c + n < q.n) to[n] = v.e[n];
        }
    } else {
        store_tile<T, PAIRS, false>(C, ws + W_X, q.Lp, i * T, k * T);
        store_tile<T, PAIRS, true>(C, ws + w_xt(q.sp, q.Lp, ap.xt ^ 1), q.sp, k * T, i * T);
    }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
struct Group {
    Table tb;
    int entry[OM], first[OM];  // of the list, and the first matrix of its batch
    size_t bytes, sums;        // of the workspace, and where the sums of split products begin
};

long long up(long long n, long long k) { return (n + k - 1) / k * k; }

long long sym_count(const Table& tb, int T) {  // tiles of one product
    long long n = 0;
    for (int i = 0; i < tb.count; ++i) {
        const long long t = tb.mat[i].sp / T;
        n += t * (t + 1) / 2 * tb.mat[i].batch;
    }
    return n;
}

// How a launch of n tiles goes to SLOTS places, two a CU: rounds of whole tiles, and
// the rest split over K (in at most so many parts) so that it fills them once
// more.  Tiles of 128 take them all at once.  Tiles of 64 of pairs, with 128 KB of
// LDS each, are one a CU and go in two rounds (448 of them take 18 us, 224 11).
struct Cut {
    int whole, parts;
};
constexpr int SLOTS = 512;
Cut cut_of(long long n, int most) {
    const int rest = (int)(n % SLOTS);
    const int parts = rest == 0 || n < SLOTS ? 1 : std::min(SLOTS / rest, most);
    return parts > 1 ? Cut{(int)n - rest, parts} : Cut{(int)n, 1};
}

// X X^T of fewer tiles than SLOTS: the longer side is often much the longer, so
// units over L of one length, of 256 at least, as many as there are places.
// Sets the entries' parts and returns all units.
long long gram_units(Table& tb, int T) {
    auto tiles = [&](const OMat& q) { const long long t = q.sp / T; return t * (t + 1) / 2 * q.batch; };
    long long cells = 0, unit = 0;  // cells: steps of 256 of L
    for (int i = 0; i < tb.count; ++i) cells += tiles(tb.mat[i]) * (up(tb.mat[i].Lp, 256) / 256);
    const long long len = std::max(1LL, (cells + SLOTS - 1) / SLOTS);
    for (int i = 0; i < tb.count; ++i) {
        OMat& q = tb.mat[i];
        q.parts = (int)std::max(1LL, up(q.Lp, 256) / 256 / len);
        q.unit0 = (int)unit;
        unit += tiles(q) * q.parts;
    }
    return unit;
}

// Tiles of 128 where they give every CU one, else of 64 (and for single tiles).
// fp32, one matrix, with the border at 100, 256 and 500 tiles: 1500 x 1500 581,
// 592, 592 us, 2048 x 2048 1025, 936, 1000, 1024 x 4096 374, 371, 414.
int tile_of(long long n128, bool fits) { return fits && n128 >= 256 ? 128 : 64; }

// The list cut into groups that share their launches and, one after the other,
// the workspace.  A group ends when its matrices alone fill the chip several
// times over, so that a long list or batch takes no more workspace than that.
std::vector<Group> groups_of(const OrthMat* mats, int count) {
    std::vector<Group> v;
    int i = 0, b = 0;  // the next matrix
    while (i < count) {
        Group g{};
        long long work = 0;
        int& n = g.tb.count;
        int unit = 64;  // of the padded sides: single tiles of 64, or tiles of either size
        while (i < count && n < OM && work < 2048) {
            const OrthMat& q = mats[i];
            OMat& o = g.tb.mat[n];
            o.s = std::min(q.m, q.n);
            o.L = std::max(q.m, q.n);
            const long long t = up(o.s, 128) / 128, one = t * (t + 1) / 2 + (up(o.s, 128) * up(o.L, 128) >> 20);
            o.batch = (int)std::min<long long>(q.batch - b, std::max(1LL, (2048 - work + one - 1) / one));
            o.ld = q.ld;
            o.ld_o = q.ld_o;
            o.bstride = q.bstride;
            o.bstride_o = q.bstride_o;
            o.m = q.m;
            o.n = q.n;
            unit = o.s > 64 ? 128 : unit;
            g.first[n] = b;
            g.entry[n++] = i;
            work += one * o.batch;
            b += o.batch;
            if (b == q.batch) {
                ++i;
                b = 0;
            }
        }
        for (int k = 0; k < n; ++k) {
            OMat& o = g.tb.mat[k];
            o.sp = (int)up(o.s, unit);
            o.Lp = (int)up(o.L, unit);
            o.ws_one = up(w_sym(o.sp, o.Lp, SYMS), 256);
            g.bytes += (size_t)(o.ws_one * o.batch);
        }
        // sums of X X^T where it is split (or left for k_orth_steps) and, where a product
        // has a remainder to split, of that
        g.sums = g.bytes;
        const long long n128 = unit == 128 ? sym_count(g.tb, 128) : 0, n64 = sym_count(g.tb, 64);
        const int T = tile_of(n128, unit == 128);
        long long cells = unit == 64 || (T == 128 ? n128 : n64) < SLOTS ? gram_units(g.tb, T) * T * T : 0;
        for (int jobs = 1; jobs <= 2; ++jobs) {
            const int t = tile_of(n128 * jobs, unit == 128);
            if ((t == 128 ? n128 : n64) * jobs >= SLOTS) cells = std::max(cells, (long long)SLOTS * t * t);
        }
        g.bytes += (size_t)cells * 4;
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

template <typename T>
struct Runner {
    static constexpr int FIRST = sizeof(T) == 4 ? PAIRS : ONES;  // how the first X is stored
    // (see the head of this file)
    static constexpr double MAX_GROWTH = sizeof(T) == 2 ? 150.0 : 12.5;
    Table& tb;
    float* sums;
    float eps;
    hipStream_t st;
    hipError_t err = hipSuccess;
    bool wide = true;    // sides are multiples of 128
    bool single = true;  // every matrix is one tile of 64
    int least_s = 1 << 30, least_L = 1 << 30;

    Runner(Group& g, char* ws, double eps_, hipStream_t s) : tb(g.tb), sums((float*)(ws + g.sums)), eps((float)eps_), st(s) {
        for (int i = 0; i < tb.count; ++i) {
            wide = wide && tb.mat[i].sp % 128 == 0 && tb.mat[i].Lp % 128 == 0;
            single = single && tb.mat[i].sp == 64;
            least_s = std::min(least_s, tb.mat[i].sp);
            least_L = std::min(least_L, tb.mat[i].Lp);
        }
    }

    template <int THREADS = WG, typename K, typename... A>
    void run(K kernel, unsigned grid, int lds, A... args) {
        if (err != hipSuccess || grid == 0) return;
        if (lds > 64 * 1024 && (err = ensure_dyn_lds((const void*)kernel, lds)) != hipSuccess) return;
        hipLaunchKernelGGL(kernel, dim3(grid), dim3(THREADS), lds, st, tb, args...);
        err = hipGetLastError();
    }

    template <int TILE, int S, bool GRAM>
    void sym_t(SymLaunch& s, int jobs) {
        constexpr int lds = product_lds<TILE, S, S>(), SLICES = TILE / JOIN_ROWS<TILE>;
        auto tiles = [](const OMat& q) { const int t = q.sp / TILE; return t * (t + 1) / 2; };
        s.sums = sums;
        s.eps = eps;
        s.tiles = (int)number(tb, tiles);
        if (GRAM && (s.tiles < SLOTS || s.leave)) {
            gram_units(tb, TILE);
            s.whole = -1;
            run<NT<TILE>>(k_orth_sym<TILE, S, GRAM>, number(tb, [&](const OMat& q) { return tiles(q) * q.parts; }), lds, s);
            if (!s.leave)
                run<NT<TILE>>(k_orth_join<TILE, GRAM>,
                              number(tb, [&](const OMat& q) { return q.parts > 1 ? tiles(q) * SLICES : 0; }), 0, s);
            return;
        }
        const Cut c = cut_of((long long)s.tiles * jobs, (GRAM ? least_L : least_s) / 256);
        s.whole = c.whole;
        s.parts = c.parts;
        const int rest = s.tiles * jobs - c.whole;
        run<NT<TILE>>(k_orth_sym<TILE, S, GRAM>, (unsigned)(c.whole + rest * c.parts), lds, s);
        if (rest) run<NT<TILE>>(k_orth_join<TILE, GRAM>, (unsigned)(rest * SLICES), 0, s);
    }
    template <int S, bool GRAM>
    void sym(SymLaunch s, int jobs = 1) {
        if (tile_of(sym_count(tb, 128) * jobs, wide) == 128) sym_t<128, S, GRAM>(s, jobs);
        else sym_t<64, S, GRAM>(s, jobs);
    }
    void products(const SymJob& a) { sym<PAIRS, false>(SymLaunch{{a, a}}); }
    void products(const SymJob& a, const SymJob& b) { sym<PAIRS, false>(SymLaunch{{a, b}}, 2); }

    template <int TILE, int S, bool LAST>
    void apply_t(const Apply& ap) {
        run<NT<TILE>>(k_orth_apply<TILE, S, T, LAST>,
                      number(tb, [](const OMat& q) { return (q.sp / TILE) * (q.Lp / TILE); }),
                      product_lds<TILE, PAIRS, S>(), ap);
    }
    template <int S, bool LAST>
    void apply(const Apply& ap) {
        long long n = 0;
        for (int i = 0; i < tb.count; ++i) n += (long long)(tb.mat[i].sp / 128) * (tb.mat[i].Lp / 128) * tb.mat[i].batch;
        if (tile_of(n, wide) == 128) apply_t<128, S, LAST>(ap);
        else apply_t<64, S, LAST>(ap);
    }
    void apply(const Apply& ap, bool last) {
        if (ap.first) last ? apply<FIRST, true>(ap) : apply<FIRST, false>(ap);
        else last ? apply<PAIRS, true>(ap) : apply<PAIRS, false>(ap);
    }

    hipError_t go(int steps, const double* coef) {
        if (!std::is_same<T, f16>::value) run(k_orth_amax<T>, number(tb, amax_wgs), 0);
        run(k_orth_prep<T>, number(tb, prep_wgs), 0);
        double lambda = 1.0;
        int xt = 0, ex = 0, step = 0;  // X is stored times 2^ex (and 1 / norm_factor in the first block)
        for (bool first = true; step < steps; first = false) {
            int len = 0;
            double growth = 1.0, l = lambda;
            while (step + len < steps && len < STEP_MAX && (len == 0 || growth <= MAX_GROWTH)) {
                const Bound b = bound_of(coef + 3 * (step + len), l);
                growth *= b.p * b.p;
                l = b.lambda;
                ++len;
            }
            const bool last = step + len == steps;
            int ea = exponent(lambda);
            SymLaunch gram{{{0, 0, 0, -1, pow2(ea - 2 * ex), 0.0f, 0.0f}, {}}};
            gram.first = first;
            gram.leave = single;
            Steps list{};
            if (first) sym<FIRST, true>(gram);
            else sym<PAIRS, true>(gram);
            int Q = -1, eq = 0;  // Q: which of the workspace's matrices 2, 3, 4
            double qb = 1.0;
            for (int k = 0; k < len; ++k, ++step) {
                const double* c = coef + 3 * step;
                const Bound b = bound_of(c, lambda);
                const int ep = exponent(b.p), et = exponent(b.p * lambda), en = exponent(b.lambda);
                const int P = Q == 2 ? 3 : 2, Q2 = Q < 0 ? P : 9 - Q - P;
                qb = std::min(qb * b.p, 1e30);
                const int eq2 = Q < 0 ? ep : exponent(qb);
                const SymJob jp{0, 0, P, 0, (float)(c[2] * pow2(ep - 2 * ea)), (float)(c[1] * pow2(ep - ea)),
                                (float)(c[0] * pow2(ep))};
                const SymJob jt{P, 0, 1, -1, pow2(et - ep - ea), 0.0f, 0.0f};
                const SymJob ja{1, P, 0, -1, pow2(en - et - ep), 0.0f, 0.0f};
                const SymJob jq{P, Q, Q2, -1, pow2(eq2 - ep - eq), 0.0f, 0.0f};
                if (single) {
                    list.one[k] = {jp.alpha, jp.beta, jp.gamma, jt.alpha, ja.alpha, jq.alpha};
                } else {
                    products(jp);
                    if (k + 1 < len) {
                        if (Q < 0) products(jt);
                        else products(jt, jq);
                        products(ja);
                    } else if (Q >= 0) {
                        products(jq);
                    }
                }
                eq = eq2;
                Q = Q2;
                ea = en;
                lambda = b.lambda;
            }
            if (single) {
                list.len = len;
                list.first = first;
                list.Q = Q;
                list.a0 = gram.job[0].alpha;
                list.eps = eps;
                list.sums = sums;
                run<512>(k_orth_steps, number(tb, [](const OMat&) { return 1; }), STEPS_LDS, list);
            }
            const int ex2 = exponent(sqrt(lambda));
            apply(Apply{Q, xt, first, pow2((last ? 0 : ex2) - eq - ex), eps}, last);
            xt ^= 1;
            ex = ex2;
        }
        return err;
    }
};

template <typename T>
hipError_t orth_t(const OrthMat* mats, int count, int steps, const double* coef, double eps, Ws ws, hipStream_t st) {
    for (Group& g : groups_of(mats, count)) {
        char* at = (char*)ws.p;
        for (int k = 0; k < g.tb.count; ++k) {
            OMat& o = g.tb.mat[k];
            const OrthMat& q = mats[g.entry[k]];
            o.g = (const T*)q.g + g.first[k] * q.bstride;
            o.o = (T*)q.o + g.first[k] * q.bstride_o;
            o.scaled = !std::is_same<T, f16>::value;
            o.ws = at;
            at += o.ws_one * o.batch;
            constexpr long long V = 16 / sizeof(T);
            auto aligned = [](const void* p, long long ld, long long stride) {
                return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % V == 0 && stride % V == 0;
            };
            // (a single row needs no distance)
            o.vec = (aligned(o.g, o.m > 1 ? o.ld : 0, o.bstride) ? 1 : 0) |
                    (aligned(o.o, o.m > 1 ? o.ld_o : 0, o.bstride_o) ? 2 : 0);
        }
        const hipError_t e = Runner<T>(g, (char*)ws.p, eps, st).go(steps, coef);
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
