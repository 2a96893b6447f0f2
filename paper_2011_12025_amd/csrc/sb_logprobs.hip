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
#include <limits.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

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

// The maximum or the sum of the lanes' values, in a fixed order, by DPP: prefixes of
// rows of 16 lanes, then of the rows; `none` where a lane has no neighbour.
template <bool MAX>
__device__ __forceinline__ float wave_total(float v, float none) {
    auto step = [&](auto ctrl, auto rows) {
        const float o = __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(none), __float_as_int(v),
                                                                   decltype(ctrl)::value, decltype(rows)::value, 0xF, false));
        v = MAX ? fmaxf(v, o) : v + o;
    };
    constexpr std::integral_constant<int, 0xF> all{};
    step(std::integral_constant<int, 0x111>{}, all);  // row_shr 1, 2, 4, 8
    step(std::integral_constant<int, 0x112>{}, all);
    step(std::integral_constant<int, 0x114>{}, all);
    step(std::integral_constant<int, 0x118>{}, all);
    step(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xA>{});  // row_bcast 15, 31
    step(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xC>{});
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

__device__ __forceinline__ Acc wave_join(Acc a) {
    const float m = wave_total<true>(a.m, LOWEST);
    raise(a, m);
    return Acc{m, wave_total<false>(a.s, 0.0f), wave_total<false>(a.t, 0.0f)};
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

// What a row's results come from.
struct Row {
    float m, ln_s;  // s = 0 (every class at -inf): an empty row
    bool empty;
    __device__ __forceinline__ explicit Row(const Acc& a) : m(a.m), ln_s(logf(a.s)), empty(a.s == 0.0f) {}
    __device__ __forceinline__ float logp(float z) const { return empty ? -INFINITY : (z - m) - ln_s; }
    __device__ __forceinline__ float lse() const { return empty ? -INFINITY : m + ln_s; }
    __device__ __forceinline__ float entropy(const Acc& a) const { return empty ? 0.0f : ln_s - LN2 * a.t / a.s; }
};

// ---------------------------------------------------------------------------
// A wave's list of alternatives: lane i holds the i-th largest key so far.
// ---------------------------------------------------------------------------
__device__ __forceinline__ u64 lane_key(u64 k, int lane) {
    return (u64)(uint32_t)__builtin_amdgcn_readlane((int)(k >> 32), lane) << 32 |
           (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)k, lane);
}

struct TopList {
    u64 key = 0;   // this lane's
    u64 last = 0;  // the topk-th
    // one more key a lane (0: none)
    __device__ __forceinline__ void offer(u64 k, int topk) {
        u64 in = __ballot(k > last);
        while (in) {
            const int src = __ffsll((unsigned long long)in) - 1;
            const u64 nk = lane_key(k, src);
            const u64 up = (u64)(uint32_t)__builtin_amdgcn_update_dpp(-1, (int)(key >> 32), 0x138, 0xF, 0xF, false) << 32 |
                           (uint32_t)__builtin_amdgcn_update_dpp(-1, (int)(uint32_t)key, 0x138, 0xF, 0xF, false);
            // (up: the key of the lane below, all ones in lane 0)
            key = key > nk ? key : up > nk ? nk : up;
            last = lane_key(key, topk - 1);
            in &= ~(1ull << src);
            in &= __ballot(k > last);
        }
    }
};

// ---------------------------------------------------------------------------
// Rows with many classes: NW waves share a row (or one of the parts it is
// split into), or with NW = 1 each wave of four has a row of its own.  A lane
// takes 16-byte vectors, LU of them in flight, and keeps its own (m, s, t).
//
// The alternatives come from the lanes' maxima, which the sums keep anyway: of 64
// groups of lanes the topk-th largest maximum is a score that at least topk
// classes reach, so they all lie in lanes whose own maximum does.  Few do (24 of
// 1024 for 20 alternatives of random scores); their vectors are read again, and
// the scores that reach the bound sorted into a list.  The pass over the row costs
// what it does without alternatives.
//
// PLANES: a wave takes a pixel of a plane, its classes a plane apart and one score a
// "vector".  For more alternatives than the registers of a thread hold: 36 pixels
// of 532 classes with 20 alternatives, listed in LDS by a thread a pixel, took 300 us.
// (Large maps are far from their bytes: a load takes 2 or 4 bytes of a line, and
// 256 x 512 pixels of 150 classes with 20 alternatives 250 us.)
// ---------------------------------------------------------------------------
constexpr int LU = 4;

template <typename T> constexpr int LV = 16 / (int)sizeof(T);

struct Part {  // results of a part of a row in the workspace, followed by topk keys
    float m, s, t, unused;
};
__host__ __device__ inline long long part_bytes(int topk) { return 16 + 8LL * topk; }

// The k-th largest of the lanes' values: the largest k times over where that is
// less than ranking all (about 14 instructions a time, 320 to rank).
__device__ __forceinline__ float kth_of_lanes(float m, int k) {
    if (k <= 16) {
        float left = m, top = -INFINITY;
        for (int i = 0; i < k; ++i) {
            top = wave_total<true>(left, -INFINITY);
            const int at = __ffsll((unsigned long long)__ballot(left == top)) - 1;
            left = lane_id() == at ? -INFINITY : left;
        }
        return top;
    }
    int rank = 0;
#pragma unroll 16
    for (int l = 0; l < 64; ++l) {
        const float o = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(m), l));
        rank += o > m || (o == m && l < lane_id()) ? 1 : 0;
    }
    const int at = __ffsll((unsigned long long)__ballot(rank == k - 1)) - 1;
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(m), at));
}

template <bool ENT, int V>
__device__ __forceinline__ void add_vectors(Acc& a, const float (&f)[LU][V], const float (&vm)[LU]) {
    float m2 = a.m;
#pragma unroll
    for (int u = 0; u < LU; ++u) m2 = fmaxf(m2, vm[u]);
    raise(a, m2);
    float s[2] = {}, t[2] = {};
#pragma unroll
    for (int u = 0; u < LU; ++u)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float d = (f[u][i] - m2) * LOG2E, e = exp2_(d);  // (NaN stays in e)
            s[(u + i) & 1] += e;
            if (ENT) t[(u + i) & 1] = fmaf(e, fmaxf(d, FAR), t[(u + i) & 1]);
        }
    a.s += s[0] + s[1];
    if (ENT) a.t += t[0] + t[1];
}

template <typename T, int NW, bool TOP, bool ENT, bool PLANES = false>
__global__ __launch_bounds__(NW == 1 ? 256 : NW * 64) void k_logp_rows(LogpArgs a, int parts, char* ws) {
    static_assert(!PLANES || NW == 1, "a wave a pixel");
    constexpr int V = PLANES ? 1 : LV<T>, THREADS = NW == 1 ? 256 : NW * 64;
    __shared__ float s_acc[3][NW];
    __shared__ u64 s_key[TOP && NW > 1 ? NW * 64 : 1];
    __shared__ float s_max[TOP && NW > 1 ? NW * 64 : 1];
    __shared__ float s_bound;
    __shared__ int s_n, s_nan;
    const int lane = lane_id(), wid = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wave = NW == 1 ? 0 : wid;
    const long long item = NW == 1 ? a.r0 + (long long)blockIdx.x * 4 + wid : a.r0 * parts + blockIdx.x;
    const long long r = NW == 1 ? item : item / parts;
    const int part = NW == 1 ? 0 : (int)(item - r * parts);
    if (r >= a.R) return;  // (NW = 1 alone: whole waves, and no barrier follows)
    const long long n = PLANES ? r / a.P : r, p = PLANES ? r - n * a.P : 0, P = PLANES ? a.P : 1;
    const T* z = (const T*)a.z + n * a.C_buf * P + p;

    // [0, head) and [tail, C) score by score, whole vectors between
    const int head = PLANES ? 0 : min(a.C, (int)((16 - (reinterpret_cast<uintptr_t>(z) & 15)) & 15) / (int)sizeof(T));
    const int nv = (a.C - head) / V, tail = head + nv * V;
    const int v0 = (int)((long long)nv * part / parts), v1 = (int)((long long)nv * (part + 1) / parts);
    const T* zv = z + head;

    Acc acc = nothing();
    const bool first = part == 0 && wave == 0 && head, final_ = part == parts - 1 && wave == NW - 1 && tail < a.C;
    const bool in_h = lane < head, in_t = tail + lane < a.C;
    const float fh = first && in_h ? to_f32(z[lane]) : -INFINITY, ft = final_ && in_t ? to_f32(z[tail + lane]) : -INFINITY;

    Vec<T, V> cur[LU], nxt[LU];
    constexpr int STEP = NW * 64 * LU;
    auto load = [&](Vec<T, V>(&to)[LU], int base) {
#pragma unroll
        for (int u = 0; u < LU; ++u) {
            const int v = base + u * 64 + lane;
            if constexpr (PLANES) {
                if (v < v1) to[u].e[0] = zv[v * P];
            } else {
                if (v < v1) to[u].raw = ld_nt16(zv + (long long)v * V);
            }
        }
    };
    const int begin = v0 + wave * (64 * LU);
    if (begin < v1) load(cur, begin);
    for (int base = begin; base < v1; base += STEP) {
        if (base + STEP < v1) load(nxt, base + STEP);
        float f[LU][V], vm[LU];
#pragma unroll
        for (int u = 0; u < LU; ++u) {
            const bool in = base + u * 64 + lane < v1;
#pragma unroll
            for (int i = 0; i < V; ++i) f[u][i] = in ? to_f32(cur[u].e[i]) : -INFINITY;
            vm[u] = f[u][0];
#pragma unroll
            for (int i = 1; i < V; ++i) vm[u] = fmaxf(vm[u], f[u][i]);
        }
        add_vectors<ENT, V>(acc, f, vm);
#pragma unroll
        for (int u = 0; u < LU; ++u) cur[u] = nxt[u];
    }
    const float mine = acc.m;
    if (first) add(acc, fh);
    if (final_) add(acc, ft);

    TopList top;
    if (TOP) {
        bool nan = __ballot(acc.s != acc.s) != 0;  // then the maxima say nothing
        float bound;
        if (NW > 1) {
            s_max[wave * 64 + lane] = mine;
            if (threadIdx.x == 0) s_n = s_nan = 0;
            __syncthreads();
            if (nan && lane == 0) s_nan = 1;
            if (wave == 0) {
                float m = mine;
                for (int w = 1; w < NW; ++w) m = fmaxf(m, s_max[w * 64 + lane]);
                m = kth_of_lanes(m, a.topk);
                if (lane == 0) s_bound = m;
            }
            __syncthreads();
            nan = s_nan != 0;
            bound = s_bound;
        } else {
            bound = kth_of_lanes(mine, a.topk);
        }
        // (a maximum of LOWEST may be that of nothing, or of -inf alone)
        const bool all = nan || bound <= LOWEST;
        if (all) bound = -INFINITY;
        if (first) top.offer(in_h ? key_of(fh, lane) : 0, a.topk);
        if (final_) top.offer(in_t ? key_of(ft, tail + lane) : 0, a.topk);
        const u64 lanes = all ? ~0ull : (u64)__ballot(mine >= bound);
        const int count = __popcll(lanes);
        // lane i: the i-th of these lanes
        const int below = __builtin_amdgcn_mbcnt_hi((uint32_t)(lanes >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)lanes, 0u));
        const int which = __builtin_amdgcn_ds_permute((lanes >> lane & 1 ? below : count + lane - below) * 4, lane);
        const int nt = (v1 - v0 + STEP - 1) / STEP * LU;  // vectors of a lane, at most
        const int together = nt >= 64 ? 1 : 64 / max(nt, 1);  // lanes whose vectors the wave reads at once
        for (int c0 = 0; c0 < count; c0 += together)
            for (int t0 = 0; t0 < nt; t0 += 64) {
                const int ci = c0 + (together > 1 ? lane / nt : 0), t = together > 1 ? lane % nt : t0 + lane;
                const int of = __shfl(which, min(ci, 63), 64);
                const int v = begin + t / LU * STEP + t % LU * 64 + of;
                const bool in = ci < min(count, c0 + together) && t < nt && v < v1;
                Vec<T, V> q = vzero<T, V>();
                if (in) q = PLANES ? vload<T, V>(zv + v * P) : vload<T, V>(zv + (long long)v * V);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float f = to_f32(q.e[i]);
                    const bool take = in && !(f < bound);
                    if (__ballot(take)) top.offer(take ? key_of(f, head + v * V + i) : 0, a.topk);
                }
            }
    }

    acc = wave_join(acc);
    if (NW > 1) {
        if (lane == 0) {
            s_acc[0][wave] = acc.m;
            s_acc[1][wave] = acc.s;
            s_acc[2][wave] = acc.t;
        }
        if (TOP) {  // the lists one behind the other, in any order
            const int have = __popcll(__ballot(lane < a.topk && top.key != 0));
            int at = 0;
            if (lane == 0 && have) at = atomicAdd(&s_n, have);
            at = __builtin_amdgcn_readfirstlane(at);
            if (lane < have) s_key[at + lane] = top.key;
        }
        __syncthreads();
        acc = Acc{s_acc[0][0], s_acc[1][0], s_acc[2][0]};
        for (int w = 1; w < NW; ++w) join(acc, Acc{s_acc[0][w], s_acc[1][w], s_acc[2][w]});
    }
    Part* out = parts > 1 ? (Part*)(ws + item * part_bytes(a.topk)) : nullptr;
    const Row row(acc);
    const int tid = NW == 1 ? lane : (int)threadIdx.x;
    auto alternative = [&](int i, u64 k) {
        if (out) {
            ((u64*)(out + 1))[i] = k;
        } else {
            const long long at = (n * a.topk + i) * P + p;
            a.top_logp[at] = row.logp(key_score(k));
            a.top_index[at] = key_class(k);
        }
    };
    if (TOP) {
        if (NW == 1) {
            if (lane < a.topk) alternative(lane, top.key);
        } else {  // the waves' lists: a key's place is the number of larger ones
            const int n = s_n;
            for (int i = tid; i < n; i += THREADS) {
                const u64 k = s_key[i];
                int rank = 0;
#pragma unroll 8
                for (int o = 0; o < n; ++o) rank += s_key[o] > k ? 1 : 0;
                if (rank < a.topk) alternative(rank, k);
            }
            // (a part may have fewer classes than topk: keys 0)
            for (int i = n + tid; i < a.topk; i += THREADS) alternative(i, 0);
        }
    }
    if (tid != 0) return;
    if (out) {
        *out = Part{acc.m, acc.s, acc.t, 0.0f};
        return;
    }
    a.lse[r] = row.lse();
    if (ENT) a.entropy[r] = row.entropy(acc);
    if (a.labels) {
        const long long t = a.labels[r];
        a.logp[r] = t == a.ignore ? 0.0f : t < 0 || t >= a.C ? NAN : row.logp(to_f32(z[t * P]));
    }
}

// The parts of a row, one workgroup a row.
constexpr int MAX_PARTS = 16;
template <typename T>
__global__ __launch_bounds__(256) void k_logp_join(LogpArgs a, int parts, const char* ws) {
    __shared__ u64 s_key[MAX_PARTS * 64];
    const long long r = blockIdx.x, pb = part_bytes(a.topk);
    const char* in = ws + r * parts * pb;
    const int n = parts * a.topk, tid = (int)threadIdx.x;
    for (int i = tid; i < n; i += 256) s_key[i] = ((const u64*)(in + i / a.topk * pb + 16))[i % a.topk];
    __syncthreads();
    Acc acc = nothing();
    for (int p = 0; p < parts; ++p) {
        const Part q = *(const Part*)(in + p * pb);
        join(acc, Acc{q.m, q.s, q.t});
    }
    const Row row(acc);
    for (int i = tid; i < n; i += 256) {
        const u64 k = s_key[i];
        int rank = 0;
        for (int o = 0; o < n; ++o) rank += s_key[o] > k ? 1 : 0;
        if (k && rank < a.topk) {
            a.top_logp[r * a.topk + rank] = row.logp(key_score(k));
            a.top_index[r * a.topk + rank] = key_class(k);
        }
    }
    if (tid == 0) {
        a.lse[r] = row.lse();
        if (a.entropy) a.entropy[r] = row.entropy(acc);
        if (a.labels) {
            const long long t = a.labels[r];
            a.logp[r] = t == a.ignore ? 0.0f
                        : t < 0 || t >= a.C ? NAN : row.logp(to_f32(((const T*)a.z)[r * a.C_buf + t]));
        }
    }
}

// ---------------------------------------------------------------------------
// One thread a row (or a few waves, each with a range of its classes): scores
// come eight at a time, the alternatives (K <= 16) are a sorted list in registers.
// Used where rows are short or where neighbouring rows are
// neighbours in memory (the pixels of a plane).
// ---------------------------------------------------------------------------
// Order of two scores as integers; INT_MIN is below all.
__device__ __forceinline__ int rank_of(float z) {
    const int b = __float_as_int(z + 0.0f);
    return z != z ? 0x7FFFFFFF : b ^ ((b >> 31) & 0x7FFFFFFF);
}
__device__ __forceinline__ float rank_score(int k) {
    return k == 0x7FFFFFFF ? NAN : __int_as_float(k ^ ((k >> 31) & 0x7FFFFFFF));
}

template <int K>
struct RegTop {  // classes come in rising order: an equal score stays behind
    int k[K], j[K];
    __device__ __forceinline__ RegTop() {
#pragma unroll
        for (int i = 0; i < K; ++i) {
            k[i] = INT_MIN;
            j[i] = 0;
        }
    }
    __device__ __forceinline__ void put(int key, int cls) {
        if (key > k[K - 1]) {
#pragma unroll
            for (int i = K - 1; i > 0; --i) {
                const bool here = key > k[i], above = key > k[i - 1];
                k[i] = above ? k[i - 1] : here ? key : k[i];
                j[i] = above ? j[i - 1] : here ? cls : j[i];
            }
            if (key > k[0]) {
                k[0] = key;
                j[0] = cls;
            }
        }
    }
    __device__ __forceinline__ int key(int i) const {
        int r = k[0];
#pragma unroll
        for (int x = 1; x < K; ++x) r = i == x ? k[x] : r;
        return r;
    }
    __device__ __forceinline__ int cls(int i) const {
        int r = j[0];
#pragma unroll
        for (int x = 1; x < K; ++x) r = i == x ? j[x] : r;
        return r;
    }
};
template <>
struct RegTop<0> {
    __device__ __forceinline__ void put(int, int) {}
    __device__ __forceinline__ int key(int) const { return 0; }
    __device__ __forceinline__ int cls(int) const { return 0; }
};
template <int K, bool ENT, bool FULL, typename Get>
__device__ __forceinline__ void scan8(Get get, int c, int c1, Acc& a, RegTop<K>& top) {
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = FULL || c + i < c1 ? get(c + i) : -INFINITY;
    float m2 = a.m;
#pragma unroll
    for (int i = 0; i < 8; ++i) m2 = fmaxf(m2, f[i]);
    raise(a, m2);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (!FULL && c + i >= c1) break;
        const float d = (f[i] - m2) * LOG2E, e = exp2_(d);
        a.s += e;
        if (ENT) a.t = fmaf(e, fmaxf(d, FAR), a.t);
        if (K != 0) top.put(rank_of(f[i]), c + i);
    }
}
template <int K, bool ENT, typename Get>
__device__ __forceinline__ void scan(Get get, int c0, int c1, Acc& a, RegTop<K>& top) {
    int c = c0;
    for (; c + 8 <= c1; c += 8) scan8<K, ENT, true>(get, c, c1, a, top);
    if (c < c1) scan8<K, ENT, false>(get, c, c1, a, top);
}

// Results of row r = n P + p; zt: the score of its label (where it has one).
template <int K, bool ENT, typename Get>
__device__ __forceinline__ void row_out(const LogpArgs& a, long long r, long long n, long long p, const Acc& acc,
                                        const RegTop<K>& top, Get get) {
    const Row row(acc);
    a.lse[r] = row.lse();
    if (ENT) a.entropy[r] = row.entropy(acc);
    if (a.labels) {
        const long long t = a.labels[r];
        a.logp[r] = t == a.ignore ? 0.0f : t < 0 || t >= a.C ? NAN : row.logp(get((int)t));
    }
    if (K != 0)
        for (int i = 0; i < a.topk; ++i) {
            const long long q = (n * a.topk + i) * a.P + p;
            a.top_logp[q] = row.logp(rank_score(top.key(i)));
            a.top_index[q] = top.cls(i);
        }
}

// Where byte f of staged rows lies in LDS: 16 bytes of room after every 128, so
// that rows at distances which are multiples of the banks do not collide.
__device__ __forceinline__ int staged(int f) { return f + (f >> 7 << 4); }
__host__ __device__ constexpr int staged_bytes(int n) { return n + n / 128 * 16 + 16; }

// The first n elements from src, as they lie there, to LDS (all threads).
template <typename T>
__device__ __forceinline__ void stage_in(const T* src, int n, char* lds) {
    constexpr int V = LV<T>;
    const int tid = (int)threadIdx.x, nt = (int)blockDim.x;
    if ((reinterpret_cast<uintptr_t>(src) & 15) == 0) {
        const int nv = n / V;
        for (int v = tid; v < nv; v += nt) *(uint4*)(lds + staged(v * 16)) = ld_nt16(src + (long long)v * V);
        for (int e = nv * V + tid; e < n; e += nt) *(T*)(lds + staged(e * (int)sizeof(T))) = src[e];
    } else {
        for (int e = tid; e < n; e += nt) *(T*)(lds + staged(e * (int)sizeof(T))) = src[e];
    }
}

// Short rows (NHWC, tokens): a workgroup stages blockDim rows as they lie and
// each thread goes through one.
template <typename T, int K, bool ENT>
__global__ __launch_bounds__(256) void k_logp_short(LogpArgs a) {
    extern __shared__ __align__(16) char lds[];
    const int tid = (int)threadIdx.x, rows = (int)blockDim.x;
    const long long r0 = (long long)blockIdx.x * rows;
    const int nr = (int)min((long long)rows, a.R - r0), ld = (int)a.C_buf;
    stage_in((const T*)a.z + r0 * ld, (nr - 1) * ld + a.C, lds);
    __syncthreads();
    if (tid >= nr) return;
    const int at = tid * ld * (int)sizeof(T);
    auto get = [&](int c) { return to_f32(*(const T*)(lds + staged(at + c * (int)sizeof(T)))); };
    Acc acc = nothing();
    RegTop<K> top;
    scan<K, ENT>(get, 0, a.C, acc, top);
    row_out<K, ENT>(a, r0 + tid, r0 + tid, 0, acc, top, get);
}

// Pixels of planes (NCHW): 64 neighbouring pixels a wave; NW waves share them
// and split the classes, so that small maps fill the chip too.
template <typename T, int K, bool ENT, int NW>
__global__ __launch_bounds__(NW == 1 ? 256 : NW * 64) void k_logp_planes(LogpArgs a) {
    extern __shared__ __align__(16) char lds[];  // the waves' results
    const int lane = lane_id(), wid = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wave = NW == 1 ? 0 : wid;
    const long long r = ((long long)blockIdx.x * (NW == 1 ? 4 : 1) + (NW == 1 ? wid : 0)) * 64 + lane;
    const bool in = r < a.R;
    const long long rr = in ? r : a.R - 1, n = rr / a.P, p = rr - n * a.P;
    const T* z = (const T*)a.z + n * a.C_buf * a.P + p;
    auto get = [&](int c) { return to_f32(z[c * a.P]); };
    Acc acc = nothing();
    RegTop<K> top;
    scan<K, ENT>(get, (int)((long long)a.C * wave / NW), (int)((long long)a.C * (wave + 1) / NW), acc, top);
    if constexpr (NW > 1) {
        float* res = (float*)lds;            // [wave][3][64]
        int* keys = (int*)(res + NW * 192);  // [wave][topk][2][64]
        res[wave * 192 + lane] = acc.m;
        res[wave * 192 + 64 + lane] = acc.s;
        res[wave * 192 + 128 + lane] = acc.t;
        if (K > 0)
#pragma unroll
            for (int i = 0; i < (K > 0 ? K : 1); ++i)
                if (i < a.topk) {
                    keys[((wave * a.topk + i) * 2) * 64 + lane] = top.key(i);
                    keys[((wave * a.topk + i) * 2 + 1) * 64 + lane] = top.cls(i);
                }
        __syncthreads();
        if (wave != 0) return;
        for (int w = 1; w < NW; ++w) {
            join(acc, Acc{res[w * 192 + lane], res[w * 192 + 64 + lane], res[w * 192 + 128 + lane]});
            if (K != 0)
                for (int i = 0; i < a.topk; ++i) {
                    const int* q = keys + ((w * a.topk + i) * 2) * 64 + lane;
                    if (q[0] != INT_MIN) top.put(q[0], q[64]);
                }
        }
    }
    if (in) row_out<K, ENT>(a, r, n, p, acc, top, get);
}

// ---------------------------------------------------------------------------
// Gradient
// ---------------------------------------------------------------------------
// Up to K alternatives in registers (class -1: none), which may name a class twice.
// K = 0: there are none; K < 0: more than that, read where they are needed.
template <int K>
struct Alts {
    int j[K > 0 ? K : 1];
    float g[K > 0 ? K : 1];
};

struct GradRow {
    float m, ln_s, g, G, gh, H;
    int label;  // -1: none
    bool empty;

    template <int K>
    __device__ __forceinline__ GradRow(const LogpGradArgs& a, long long r, long long n, long long p, Alts<K>& alts) {
        m = a.lse[r];
        ln_s = 0.0f;
        empty = m == -INFINITY;
        g = 0.0f;
        label = -1;
        if (a.d_logp) {
            const long long l = a.labels[r];
            const bool in = l >= 0 && l < a.C;
            if (l != a.ignore) {
                label = in ? (int)l : -1;
                g = in ? a.d_logp[r] : NAN;
            }
        }
        gh = a.d_entropy ? a.d_entropy[r] : 0.0f;
        H = a.d_entropy ? a.entropy[r] : 0.0f;
        G = g;
        auto take = [&](long long q, int& j, float& d) {
            j = a.top_index[q];
            d = a.d_top[q];
            G += j < 0 || j >= a.C ? NAN : d;
        };
        if constexpr (K > 0) {
#pragma unroll
            for (int u = 0; u < K; ++u) {
                alts.j[u] = -1;
                alts.g[u] = 0.0f;
                if (u < a.topk) take((n * a.topk + u) * a.P + p, alts.j[u], alts.g[u]);
            }
        } else if constexpr (K < 0) {
            int j;
            float d;
#pragma unroll 8
            for (int i = 0; i < a.topk; ++i) take((n * a.topk + i) * a.P + p, j, d);
        }
    }
    // p from lse is off by |lse| 2^-25: past 256 it comes from the row's own maximum
    __device__ __forceinline__ bool far() const { return !empty && !(fabsf(m) <= 256.0f); }
    __device__ __forceinline__ void take(const Acc& acc) {
        const Row row(acc);
        m = row.m;
        ln_s = row.ln_s;
    }
    // what every class gets
    __device__ __forceinline__ float all(float z) const {
        const float lp = (z - m) - ln_s, pr = exp2_(lp * LOG2E);
        const float d = -pr * (G + gh * (fmaxf(lp, FAR) + H));
        return empty ? 0.0f : d;
    }
    // and the label's class or an alternative's in full
    __device__ __forceinline__ float at(const LogpGradArgs& a, float z, int j, long long n, long long p) const {
        float d = all(z);
        if (empty) return d;
        if (j == label) d += g;
#pragma unroll 8
        for (int i = 0; i < a.topk; ++i) {
            const long long q = (n * a.topk + i) * a.P + p;
            const float gi = a.d_top[q];  // (read either way: the loads of several go out together)
            d += a.top_index[q] == j ? gi : 0.0f;
        }
        return d;
    }
    // The same with alternatives in registers (K <= 0: the label alone).
    template <int K>
    __device__ __forceinline__ float at(const Alts<K>& alts, float z, int c) const {
        float d = all(z);
        if (empty) return d;
        d += c == label ? g : 0.0f;
        if constexpr (K > 0)
#pragma unroll
            for (int u = 0; u < K; ++u) d += c == alts.j[u] ? alts.g[u] : 0.0f;
        return d;
    }
    // More of them than registers hold, in [c0, c1) by one thread after the rest: eight
    // at a time against the whole list (each for itself, 20 alternatives of 10000
    // pixels took 34 us, mostly round trips to the list, and so 21).
    template <typename Get, typename Put>
    __device__ __forceinline__ void again(const LogpGradArgs& a, long long n, long long p, int c0, int c1, Get get, Put put) const {
        if (empty) return;
        for (int i0 = 0; i0 < a.topk; i0 += 8) {
            int j[8];
            float d[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                j[u] = a.top_index[(n * a.topk + min(i0 + u, a.topk - 1)) * a.P + p];  // (the last one again: the same value)
                d[u] = j[u] == label ? g : 0.0f;
            }
#pragma unroll 8
            for (int i = 0; i < a.topk; ++i) {
                const long long q = (n * a.topk + i) * a.P + p;
                const int ji = a.top_index[q];
                const float gi = a.d_top[q];
#pragma unroll
                for (int u = 0; u < 8; ++u) d[u] += ji == j[u] ? gi : 0.0f;
            }
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (j[u] >= c0 && j[u] < c1) put(j[u], all(get(j[u])) + d[u]);
        }
    }
};

// A range of a long row a workgroup.
template <typename T>
__global__ __launch_bounds__(256) void k_logp_grad_rows(LogpGradArgs a, int chunks, int per) {
    constexpr int V = LV<T>;
    const unsigned row_in = blockIdx.x / (unsigned)chunks;
    const long long r = a.r0 + row_in;
    const int chunk = (int)(blockIdx.x - row_in * chunks), tid = (int)threadIdx.x;
    const T* z = (const T*)a.z + r * a.C_buf;
    T* dz = (T*)a.dz + r * a.C_dbuf;
    Alts<-1> none;
    GradRow row(a, r, r, 0, none);
    if (row.far()) {
        __shared__ float s[3][4];
        Acc acc = nothing();
        for (int j = tid; j < a.C; j += 256) add(acc, to_f32(z[j]));
        acc = wave_join(acc);
        if (lane_id() == 0) {
            s[0][tid >> 6] = acc.m;
            s[1][tid >> 6] = acc.s;
            s[2][tid >> 6] = acc.t;
        }
        __syncthreads();
        acc = Acc{s[0][0], s[1][0], s[2][0]};
        for (int w = 1; w < 4; ++w) join(acc, Acc{s[0][w], s[1][w], s[2][w]});
        row.take(acc);
    }
    // vectors where both rows begin alike
    const int mis = (int)(reinterpret_cast<uintptr_t>(dz) & 15);
    const bool vec = mis == (int)(reinterpret_cast<uintptr_t>(z) & 15);
    const int head = vec ? min(a.C, ((16 - mis) & 15) / (int)sizeof(T)) : a.C;
    const int nv = (a.C - head) / V, tail = head + nv * V;
    const int c0 = chunk * per, c1 = min(a.C, c0 + per);
    auto single = [&](int j0, int j1) {
        for (int j = max(j0, c0) + tid; j < min(j1, c1); j += 256) dz[j] = from_f32<T>(row.all(to_f32(z[j])));
    };
    single(0, head);
    single(tail, a.C);
    // the vectors that begin in [c0, c1)
    const int v0 = min(nv, max(0, (c0 - head + V - 1) / V)), v1 = min(nv, max(0, (c1 - head + V - 1) / V));
    const int vs = c0 <= head ? 0 : v0;
#pragma unroll 4
    for (int v = vs + tid; v < v1; v += 256) {
        Vec<T, V> q, o;
        q.raw = ld_nt16(z + head + (long long)v * V);
#pragma unroll
        for (int i = 0; i < V; ++i) o.e[i] = from_f32<T>(row.all(to_f32(q.e[i])));
        st_nt16(dz + head + (long long)v * V, o.raw);
    }
    // the label's class and the alternatives again, once the rest is written
    __syncthreads();
    if (tid <= a.topk) {
        const int j = tid < a.topk ? a.top_index[r * a.topk + tid] : row.label;
        // (the workgroup that wrote it: a vector belongs to the range it begins in)
        const int first = j < head || j >= tail ? j : head + (j - head) / V * V;
        if (j >= 0 && j < a.C && first >= c0 && first < c1) dz[j] = from_f32<T>(row.at(a, to_f32(z[j]), j, r, 0));
    }
}

// Short rows, as k_logp_short: gradients go through LDS too, at `out`.
template <typename T, int K>
__global__ __launch_bounds__(256) void k_logp_grad_short(LogpGradArgs a, int out) {
    extern __shared__ __align__(16) char lds[];
    const int tid = (int)threadIdx.x, rows = (int)blockDim.x;
    const long long r0 = (long long)blockIdx.x * rows;
    const int nr = (int)min((long long)rows, a.R - r0), ld = (int)a.C_buf;
    stage_in((const T*)a.z + r0 * ld, (nr - 1) * ld + a.C, lds);
    __syncthreads();
    if (tid < nr) {
        const long long r = r0 + tid;
        const int at = tid * ld * (int)sizeof(T), to = tid * a.C * (int)sizeof(T);
        auto get = [&](int c) { return to_f32(*(const T*)(lds + staged(at + c * (int)sizeof(T)))); };
        auto put = [&](int c, float v) { *(T*)(lds + out + staged(to + c * (int)sizeof(T))) = from_f32<T>(v); };
        Alts<K> alts;
        GradRow row(a, r, r, 0, alts);
        if (row.far()) {
            Acc acc = nothing();
            RegTop<0> none;
            scan<0, false>(get, 0, a.C, acc, none);
            row.take(acc);
        }
#pragma unroll 4
        for (int c = 0; c < a.C; ++c) put(c, row.all(get(c)));
        if (row.label >= 0) put(row.label, row.at(alts, get(row.label), row.label));
        if constexpr (K > 0) {
#pragma unroll
            for (int u = 0; u < K; ++u)
                if (alts.j[u] >= 0 && alts.j[u] < a.C) put(alts.j[u], row.at(alts, get(alts.j[u]), alts.j[u]));
        } else if constexpr (K < 0) {
            row.again(a, r, 0, 0, a.C, get, put);
        }
    }
    __syncthreads();
    T* dz = (T*)a.dz + r0 * a.C_dbuf;
    const int n = nr * a.C;
    auto held = [&](int e) { return *(const T*)(lds + out + staged(e * (int)sizeof(T))); };
    if (a.C_dbuf == a.C && (reinterpret_cast<uintptr_t>(dz) & 15) == 0) {
        constexpr int V = LV<T>;
        const int nv = n / V;
        for (int v = tid; v < nv; v += rows) st_nt16(dz + (long long)v * V, *(const uint4*)(lds + out + staged(v * 16)));
        for (int e = nv * V + tid; e < n; e += rows) dz[e] = held(e);
    } else {
        for (int e = tid; e < n; e += rows) {
            const int q = e / a.C;
            dz[q * a.C_dbuf + (e - q * a.C)] = held(e);
        }
    }
}

// Pixels of planes: a thread a pixel and range of classes.  The label and the
// alternatives are looked for at every class, since a second write to a class here
// and there costs more (4 x 256 x 512 pixels of 19 fp32 classes, no, one and three
// alternatives: 24, 60 and 72 us, and so 15, 16 and 18).
template <typename T, int K>
__global__ __launch_bounds__(256) void k_logp_grad_planes(LogpGradArgs a, int per) {
    const long long r = (long long)blockIdx.x * 256 + threadIdx.x;
    if (r >= a.R) return;
    const long long n = r / a.P, p = r - n * a.P;
    const T* z = (const T*)a.z + n * a.C_buf * a.P + p;
    T* dz = (T*)a.dz + n * a.C_dbuf * a.P + p;
    const int c0 = (int)blockIdx.y * per, c1 = min(a.C, c0 + per);
    auto get = [&](int c) { return to_f32(z[c * a.P]); };
    Alts<K> alts;
    GradRow row(a, r, n, p, alts);
    if (row.far()) {
        Acc acc = nothing();
        RegTop<0> none;
        scan<0, false>(get, 0, a.C, acc, none);
        row.take(acc);
    }
#pragma unroll 8
    for (int c = c0; c < c1; ++c) dz[c * a.P] = from_f32<T>(row.at(alts, get(c), c));
    if constexpr (K < 0) row.again(a, n, p, c0, c1, get, [&](int c, float v) { dz[c * a.P] = from_f32<T>(v); });
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
// Rows for one thread each: short ones, staged as they lie (with the channels
// of the buffer that are no classes), past 64 classes where they are many (bf16, a
// thread and a wave a row: 60000 x 100 11 us and over 50, 8192 x 100 14.6 and 13.4).
// Returns rows of a workgroup, or 0.
int short_rows(int es, long long R, int C, long long ld, bool grad) {
    if (ld > 2LL * C || C > 128 || (C > 64 && R < 16384)) return 0;
    // (a workgroup takes fewer where all would leave CUs idle)
    for (int rows = R >= 65536 ? 256 : R >= 32768 ? 128 : 64; rows >= 64; rows /= 2)
        if (staged_bytes((int)std::min<long long>(rows * ld * es, 1 << 20)) + (grad ? staged_bytes(rows * C * es) : 0) <=
            (rows == 64 ? 48 : 24) * 1024)
            return rows;
    return 0;
}

// Waves of a row.  One, four of them a workgroup, where the rows fill the chip
// and are at most 16 KB (4096 rows, one and four waves: 2048 bf16 classes 6.0 and
// 12.1 us, 8192 18.3 and 19.2, fp32 8192 23.1 and 21.8), sixteen for few long ones
// (256 x 50001 bf16: 10.9, with four 19.6).
int row_waves(int es, long long R, int C) {
    if (C <= 1024 || (C * (long long)es <= 16384 && R >= 1024)) return 1;
    return C <= 16384 || R >= 512 ? 4 : 16;
}

// Parts of a long row where the rows alone leave most of the chip idle (131072 bf16
// classes, split and not: one row 11.2 and 19.7 us, 32 rows 17.7 and 21.7; 65536
// 13.0 and 14.3, 32000 12.6 and 11.3).
int row_parts(long long R, int C) {
    if (C < 65536 || R >= 64) return 1;
    return (int)std::min<long long>({MAX_PARTS, C / 16384, 256 / R});
}

// Whether a thread keeps the alternatives in registers (else a wave a row sorts
// them): 16 of them cost 80 instructions a class, which a short row has few of.
bool reg_top(int topk, int C) { return topk <= 8 || (topk <= 16 && C <= 64); }

bool is_planes(long long P) { return P > 1; }

template <typename T, int K>
hipError_t logp_k(const LogpArgs& a, hipStream_t st, int rows, bool planes) {
    const bool ent = a.entropy != nullptr;
    const int es = sizeof(T);
    if (!planes) {
        const int lds = staged_bytes(((rows - 1) * (int)a.C_buf + a.C) * es + 16);
        const unsigned grid = (unsigned)((a.R + rows - 1) / rows);
        auto run = [&](auto kernel) -> hipError_t {
            hipLaunchKernelGGL(kernel, dim3(grid), dim3(rows), lds, st, a);
            return hipGetLastError();
        };
        return ent ? run(k_logp_short<T, K, true>) : run(k_logp_short<T, K, false>);
    }
    // waves that share 64 pixels: until there are eight waves a SIMD or so
    const long long waves = (a.R + 63) / 64;
    const int nw = waves >= 4096 || a.C < 32 ? 1 : waves >= 1024 || a.C < 128 ? 4 : 16;
    auto run = [&](auto kernel, int w) -> hipError_t {
        const int all = w == 1 ? 4 : w;
        const int lds = w > 1 ? w * 768 + w * a.topk * 512 : 0;
        const unsigned grid = (unsigned)(w == 1 ? (waves + 3) / 4 : waves);
        if (lds > 64 * 1024)
            if (hipError_t e = ensure_dyn_lds((const void*)kernel, lds); e != hipSuccess) return e;
        hipLaunchKernelGGL(kernel, dim3(grid), dim3(all * 64), lds, st, a);
        return hipGetLastError();
    };
    if (nw == 16) return ent ? run(k_logp_planes<T, K, true, 16>, 16) : run(k_logp_planes<T, K, false, 16>, 16);
    if (nw == 4) return ent ? run(k_logp_planes<T, K, true, 4>, 4) : run(k_logp_planes<T, K, false, 4>, 4);
    return ent ? run(k_logp_planes<T, K, true, 1>, 1) : run(k_logp_planes<T, K, false, 1>, 1);
}

// A launch holds less than 2^32 threads: rows with a wave or more each go in pieces.
constexpr long long MAX_THREADS = 1LL << 31;

template <typename T, int NW, bool PLANES = false>
hipError_t logp_rows(LogpArgs a, Ws ws, hipStream_t st, int parts) {
    const long long piece = MAX_THREADS / (NW * 64) / parts;
    for (; a.r0 < a.R; a.r0 += piece) {
        const long long rows = std::min(piece, a.R - a.r0), items = NW == 1 ? (rows + 3) / 4 : rows * parts;
        const dim3 grid((unsigned)items), block(NW == 1 ? 256 : NW * 64);
        auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, st, a, parts, (char*)ws.p); };
        if constexpr (PLANES)
            a.entropy ? run(k_logp_rows<T, NW, true, true, true>) : run(k_logp_rows<T, NW, true, false, true>);
        else if (a.topk) a.entropy ? run(k_logp_rows<T, NW, true, true>) : run(k_logp_rows<T, NW, true, false>);
        else a.entropy ? run(k_logp_rows<T, NW, false, true>) : run(k_logp_rows<T, NW, false, false>);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T>
hipError_t logp_t(const LogpArgs& a, Ws ws, hipStream_t st) {
    const bool planes = is_planes(a.P);
    if (planes && !reg_top(a.topk, a.C)) return logp_rows<T, 1, true>(a, ws, st, 1);
    const int rows = planes ? 0 : short_rows(sizeof(T), a.R, a.C, a.C_buf, false);
    if (planes || (rows && reg_top(a.topk, a.C))) {
        if (a.topk == 0) return logp_k<T, 0>(a, st, rows, planes);
        if (a.topk == 1) return logp_k<T, 1>(a, st, rows, planes);
        if (a.topk <= 4) return logp_k<T, 4>(a, st, rows, planes);
        return a.topk <= 8 ? logp_k<T, 8>(a, st, rows, planes) : logp_k<T, 16>(a, st, rows, planes);
    }
    const int parts = row_parts(a.R, a.C);
    if (parts > 1) {
        const hipError_t e = logp_rows<T, 4>(a, ws, st, parts);
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(k_logp_join<T>, dim3((unsigned)a.R), dim3(256), 0, st, a, parts, (const char*)ws.p);
        return hipGetLastError();
    }
    const int nw = row_waves(sizeof(T), a.R, a.C);
    if (nw == 1) return logp_rows<T, 1>(a, ws, st, 1);
    return nw == 4 ? logp_rows<T, 4>(a, ws, st, 1) : logp_rows<T, 16>(a, ws, st, 1);
}

template <typename T, int K>
hipError_t grad_k(const LogpGradArgs& a, hipStream_t st, int rows) {
    if (is_planes(a.P)) {
        const long long wgs = (a.R + 255) / 256;
        // ranges of classes until there are eight workgroups a CU
        const int ranges = (int)std::max(1LL, std::min<long long>(2048 / wgs, a.C / 16));
        const int per = (a.C + ranges - 1) / ranges;
        hipLaunchKernelGGL((k_logp_grad_planes<T, K>), dim3((unsigned)wgs, (a.C + per - 1) / per), dim3(256), 0, st, a, per);
    } else {
        const int es = sizeof(T), out = (staged_bytes(((rows - 1) * (int)a.C_buf + a.C) * es + 16) + 15) / 16 * 16;
        const int lds = out + staged_bytes(rows * a.C * es + 16);
        if (lds > 64 * 1024)
            if (hipError_t e = ensure_dyn_lds((const void*)k_logp_grad_short<T, K>, lds); e != hipSuccess) return e;
        hipLaunchKernelGGL((k_logp_grad_short<T, K>), dim3((unsigned)((a.R + rows - 1) / rows)), dim3(rows), lds, st, a, out);
    }
    return hipGetLastError();
}

template <typename T>
hipError_t grad_t(const LogpGradArgs& a, hipStream_t st) {
    const int rows = is_planes(a.P) ? 0 : short_rows(sizeof(T), a.R, a.C, a.C_buf, true);
    if (is_planes(a.P) || rows) {
        if (a.topk > 8) return grad_k<T, -1>(a, st, rows);
        if (a.topk == 0) return grad_k<T, 0>(a, st, rows);
        if (a.topk == 1) return grad_k<T, 1>(a, st, rows);
        return a.topk <= 4 ? grad_k<T, 4>(a, st, rows) : grad_k<T, 8>(a, st, rows);
    }
    // ranges of 4 vectors a thread, or 16 where rows are many
    const int per = 256 * LV<T> * (a.R * a.C >= (64LL << 20) ? 16 : 4);
    const int chunks = (int)(((long long)a.C + per - 1) / per);
    const long long piece = std::max(1LL, MAX_THREADS / 256 / chunks);
    LogpGradArgs b = a;
    for (; b.r0 < b.R; b.r0 += piece) {
        const long long rows = std::min(piece, b.R - b.r0);
        hipLaunchKernelGGL(k_logp_grad_rows<T>, dim3((unsigned)(rows * chunks)), dim3(256), 0, st, b, chunks, per);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

int logp_max_top() { return 64; }

size_t logp_ws_bytes(int dtype, const LogpArgs& a) {
    const int es = dtype == 0 ? 4 : 2;
    if (is_planes(a.P) || short_rows(es, a.R, a.C, a.C_buf, false)) return 0;
    const int parts = row_parts(a.R, a.C);
    return parts > 1 ? (size_t)(a.R * parts * part_bytes(a.topk)) : 0;
}

hipError_t launch_logp(int dtype, const LogpArgs& a, Ws ws, hipStream_t st) {
    if (dtype == 0) return logp_t<float>(a, ws, st);
    return dtype == 1 ? logp_t<f16>(a, ws, st) : logp_t<bf16>(a, ws, st);
}

hipError_t launch_logp_grad(int dtype, const LogpGradArgs& a, hipStream_t st) {
    if (dtype == 0) return grad_t<float>(a, st);
    return dtype == 1 ? grad_t<f16>(a, st) : grad_t<bf16>(a, st);
}

}  // namespace sb
