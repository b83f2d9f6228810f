// token_logprobs: log probabilities of given tokens, entropy, likeliest tokens.
//
// A row's logits are read once from memory.  Each thread keeps, of
// its own elements, the largest x, the sum of 2^d and the sum of d 2^d with d
// = (x - largest) log2(e) / tau; the workgroup joins them.  The entropy is
// ln S - (sum of d e^d) / S, both terms of one sign each, so that nothing
// cancels.
//
// The k largest: on the way, the maximum of every block of 64 elements (eight
// where rows are short) goes to LDS.  The maxima of 256 groups of blocks are 256
// different elements, so their k-th largest is a bound below which nothing can
// be among the row's k.  Only blocks that reach it, little more than k, are read
// again -- whole lines -- and what reaches it too is kept; those few are ranked
// by (order of the value, lowest index first).  Where ties or an order of the
// row let more reach it than there is room for, the row is walked in tiles, and
// the bound is raised after each.
//
// Where rows are few, several workgroups share one, each with the k largest of
// its part, and a second kernel joins them.
//
// 4096 x 32768 FP16, calls one after the other on two inputs in turn: 54 us without
// alternatives, 4.9 TB/s; 64 with 20 of them, 72 with 64: a row's sums, bound, second
// reading and ranking follow each other and hide behind other rows only, and they
// are 1000 vector instructions a row with one alternative, 3000 with 64, beside 12
// a logit, the vector ALUs' share of the stream.  Floats, twice the bytes: 92, 99
// and 105 us.  One row of 50001 floats, 20 alternatives: 9 us and 5 for the join.
#include "row_ops.h"

namespace fp8t {
namespace {

constexpr int kMaxGiven = 4096;
constexpr int64_t kAcross = 1 << 20;           // rows along a grid's first dimension
constexpr int64_t kMaxV = FP8T_MAX_VOCAB;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

struct LogprobArgs {
    const void* z;
    const int64_t* idx;
    float* logp;
    float* entropy;
    float* stats;
    int64_t* top_idx;
    float* top_logp;
    int64_t z_ld, N;
    int V, m, k, parts, per;           // workgroups of a row, elements of each
    float to2, tau;                    // to2 = log2(e) / tau
    float4* part_sums;                 // N x parts: largest, sum, sum of d 2^d
    uint64_t* part_top;                // N x parts x k
};

// Largest element (kTop for +Inf, whose distance from it is +Inf then), sum of 2^d,
// sum of d 2^d.  So s is +Inf with an element of +Inf, NaN with a NaN alone.
struct Soft {
    float m, s, t;
};
constexpr float kTop = 0x1.fffffep127f;        // FP32's largest
// The sums of x relative to m, its largest or larger.  Nothing there (-Inf) stays
// nothing, a NaN stays.
__device__ __forceinline__ void move_to(Soft& x, float m, float to2) {
    const float d = x.m == m ? 0.0f : fmaxf((x.m - m) * to2, -1000.0f), f = __builtin_amdgcn_exp2f(d);
    x.t = f * __builtin_fmaf(d, x.s, x.t);
    x.s *= f;
    x.m = m;
}
__device__ __forceinline__ Soft join(Soft a, Soft b, float to2) {
    const float m = fmaxf(a.m, b.m);
    move_to(a, m, to2);
    move_to(b, m, to2);
    a.s += b.s;
    a.t += b.t;
    return a;
}
// The sums of a wave's lanes, in all of them: the largest first, so that each
// lane's sums move once.
__device__ __forceinline__ Soft wave_join(Soft x, float to2) {
    float m = x.m;
#pragma unroll
    for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
    move_to(x, m, to2);
#pragma unroll
    for (int d = 32; d; d >>= 1) {
        x.s += __shfl_xor(x.s, d);
        x.t += __shfl_xor(x.t, d);
    }
    return x;
}

// Order of a float as a whole number: -0 is 0, NaN is above +Inf.
__device__ __forceinline__ uint32_t order_of(float x) {
    if (x != x) return 0xFFFFFFFFu;
    const uint32_t u = __float_as_uint(x + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
// (order, lowest index first): different for every element of a row.
__device__ __forceinline__ uint64_t key_of(uint32_t order, int v) {
    return ((uint64_t)order << 32) | (uint32_t)~v;
}
__device__ __forceinline__ int index_of(uint64_t key) { return (int)~(uint32_t)key; }

// keys[0, n), n <= size (a power of two), largest first; all threads.
template <int T>
__device__ __forceinline__ void sort_keys(uint64_t* keys, int n, int size) {
    for (int i = n + threadIdx.x; i < size; i += T) keys[i] = 0;
    for (int len = 2; len <= size; len <<= 1)
        for (int d = len >> 1; d; d >>= 1) {
            __syncthreads();
            for (int i = threadIdx.x; i < size / 2; i += T) {
                const int a = 2 * i - (i & (d - 1)), b = a + d;
                const uint64_t x = keys[a], y = keys[b];
                if ((x < y) == ((a & len) == 0)) {
                    keys[a] = y;
                    keys[b] = x;
                }
            }
        }
    __syncthreads();
}

// What the selection of a row's top keeps in LDS.
constexpr int kFew = 256;
template <int ROOM, int GROUPS>
struct Selection {
    static constexpr int kRoom = ROOM, kGroups = GROUPS;
    __attribute__((aligned(16))) uint64_t keys[ROOM];
    __attribute__((aligned(16))) uint64_t few[kFew];
    uint64_t top[FP8T_MAX_TOP];
    uint32_t group[GROUPS];
    uint32_t bound;
    int count, kept;
};

// A bound that at least k of the groups' maxima reach, and few more (below all
// of them where there are fewer): its bits from the first one in which the
// groups differ.  All threads; group is complete before the call.
template <int T, typename S>
__device__ __forceinline__ uint32_t find_bound(S& s, int k) {
    __syncthreads();
    constexpr int kGroups = S::kGroups;
    const int lane = threadIdx.x & 63;
    if (threadIdx.x < 64) {
        uint32_t g[kGroups / 64], hi = 0, lo = 0xFFFFFFFFu;
#pragma unroll
        for (int i = 0; i < kGroups / 64; ++i) {
            g[i] = s.group[i * 64 + lane];
            hi = max(hi, g[i]);
            lo = min(lo, g[i]);
        }
#pragma unroll
        for (int d = 32; d; d >>= 1) {
            hi = max(hi, (uint32_t)__shfl_xor((int)hi, d));
            lo = min(lo, (uint32_t)__shfl_xor((int)lo, d));
        }
        hi = __builtin_amdgcn_readfirstlane(hi);
        lo = __builtin_amdgcn_readfirstlane(lo);
        int b = hi == lo ? -1 : 31 - __clz(hi ^ lo);
        uint32_t bound = b < 0 ? lo : lo & ~((2u << b) - 1u);
        for (; b >= 0; --b) {
            const uint32_t tried = bound | (1u << b);
            int reach = 0;
#pragma unroll
            for (int i = 0; i < kGroups / 64; ++i) reach += __popcll(__ballot(g[i] >= tried));
            if (reach >= k) bound = tried;
            if (reach >= k && reach <= k + k / 8) break;
        }
        if (lane == 0) s.bound = bound;
    }
    __syncthreads();
    return s.bound;
}

// The k largest of keys[0, n) to top, each to the place that is the number of
// larger ones.
template <int T>
__device__ __forceinline__ void rank_keys(uint64_t* keys, int n, uint64_t* top, int k) {
    for (int i = n + threadIdx.x; i < ((n + 7) & ~7); i += T) keys[i] = 0;
    __syncthreads();
#pragma unroll 1
    for (int own = threadIdx.x; own < n; own += T) {
        const uint64_t mine = keys[own];
        int place = 0;
#pragma unroll 1
        for (int i = 0; i < n; i += 8)
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                const ulonglong2 two = *reinterpret_cast<const ulonglong2*>(keys + i + j);
                place += (int)(two.x > mine) + (int)(two.y > mine);
            }
        if (place < k) top[place] = mine;
    }
    __syncthreads();
}

// Where the k largest of s.keys[0, n) then are, in order; n <= S::kRoom.  All
// threads.
template <int T, typename S>
__device__ __forceinline__ const uint64_t* top_keys(S& s, int n, int k) {
    constexpr int kGroups = S::kGroups;
    const int tid = threadIdx.x;
    if (n <= 128 || n <= k + k / 2) {                       // ranking costs n squared
        rank_keys<T>(s.keys, n, s.top, k);
        return s.top;
    }
    // fewer first: those that reach the k-th largest of the groups
    for (int g = tid; g < kGroups; g += T) {
        uint32_t top = 0;
        for (int i = g; i < n; i += kGroups) top = max(top, (uint32_t)(s.keys[i] >> 32));
        s.group[g] = top;
    }
    if (tid == 0) s.kept = 0;
    const uint32_t bound = find_bound<T>(s, k);
    for (int i = tid; i < n; i += T)
        if ((uint32_t)(s.keys[i] >> 32) >= bound) {
            const int at = atomicAdd(&s.kept, 1);
            if (at < kFew) s.few[at] = s.keys[i];
        }
    __syncthreads();
    if (s.kept <= kFew) {
        rank_keys<T>(s.few, s.kept, s.top, k);
        return s.top;
    }
    int size = 2;                                           // ties
    while (size < n) size <<= 1;
    sort_keys<T>(s.keys, n, size);
    return s.keys;
}

template <int FZ>
__device__ __forceinline__ Eight<FZ> load_logits(const fmt_t<FZ>* row, int v, int V) {
    if (v + 8 <= V) return *reinterpret_cast<const Eight<FZ>*>(row + v);
    Eight<FZ> e;                                            // -Inf past the end
    if constexpr (FZ == FP8T_FMT_F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            e.a[i] = v + i < V ? row[v + i] : -INFINITY;
            e.b[i] = v + 4 + i < V ? row[v + 4 + i] : -INFINITY;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t lo = v + 2 * i < V ? row[v + 2 * i] : 0xFE00u;
            const uint32_t hi = v + 2 * i + 1 < V ? row[v + 2 * i + 1] : 0xFE00u;
            e.a[i] = lo | (hi << 16);
        }
    }
    return e;
}

// Logits as the sums take them: times 2^-96 from FP16 (the codes' fields moved
// into a float's, one instruction less), as they are from floats.  Values that
// are not finite come out as finite FP16 ones of 2^32 and more.
template <int FZ>
struct Raw {
    static constexpr float kUnit = FZ == FP8T_FMT_FP16 ? 0x1p96f : 1.0f;
    __device__ static __forceinline__ void values(const Eight<FZ>& e, float* y) {
        if constexpr (FZ == FP8T_FMT_F32) {
            values8<FZ>(e, y);
        } else {
            float top = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                y[2 * i] = __uint_as_float((uint32_t)((int32_t)(e.a[i] << 16) >> 2) & 0x9FFFC000u);
                y[2 * i + 1] = __uint_as_float((uint32_t)((int32_t)e.a[i] >> 2) & 0x9FFFC000u);
                top = max3_abs(top, y[2 * i], y[2 * i + 1]);
            }
            if (__builtin_expect(top >= 0x1p-64f, 0)) {
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = fp16_to_f32((e.a[i / 2] >> (16 * (i % 2))) & 0xFFFFu) * 0x1p-96f;
            }
        }
    }
};
// The largest of three in one instruction (fmaxf of values from bits takes three),
// a NaN left out.
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
// Constants of the loops over logits.  In vector registers: instructions that
// read scalar ones issue at half rate.
struct Consts {
    float to2, unit;
    __device__ __forceinline__ Consts(float to2_, float unit_)
        : to2(__uint_as_float(in_vgpr(__float_as_uint(to2_)))),
          unit(__uint_as_float(in_vgpr(__float_as_uint(unit_)))) {}
};
constexpr float kFloor2 = -160.0f;     // below it powers are 0

// N times eight logits more: y is what Raw gives; top: the largest of each eight,
// of the same unit.
template <int FZ, int N>
__device__ __forceinline__ void add_logits(Soft& x, const float (&y)[N][8], float (&top)[N], const Consts& k) {
    float all = -INFINITY;
#pragma unroll
    for (int u = 0; u < N; ++u) {
        top[u] = max3(y[u][0], y[u][1], y[u][2]);
        top[u] = max3(top[u], y[u][3], y[u][4]);
        top[u] = max3(top[u], y[u][5], y[u][6]);
        top[u] = max3(top[u], y[u][7], y[u][7]);
        all = fmaxf(all, top[u]);
    }
    all = fminf(all * k.unit, kTop);
    if (all > x.m) move_to(x, all, k.to2);
    const float m = x.m == -INFINITY ? 0.0f : x.m;
    float s = 0.0f, t = 0.0f;                               // of these alone: shorter chains of additions
#pragma unroll
    for (int u = 0; u < N; ++u)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            // the distance first, exact or rounded once
            const float d = (FZ == FP8T_FMT_F32 ? y[u][i] - m : __builtin_fmaf(y[u][i], k.unit, -m)) * k.to2;
            const float p = __builtin_amdgcn_exp2f(d);
            s += p;
            t = __builtin_fmaf(fmaxf(d, kFloor2), p, t);     // d = -Inf adds 0
        }
    x.s += s;
    x.t += t;
}

// The largest of eight neighbouring lanes, in all of them: an instruction a step
// (three from builtins), two states after the one that wrote what other lanes
// read.
__device__ __forceinline__ float max_of_8_lanes(float x) {
    float r;
    asm("s_nop 1\n\tv_max_f32_dpp %0, %1, %1 quad_perm:[1,0,3,2] row_mask:0xf bank_mask:0xf\n\t"
        "s_nop 1\n\tv_max_f32_dpp %0, %0, %0 quad_perm:[2,3,0,1] row_mask:0xf bank_mask:0xf\n\t"
        "s_nop 1\n\tv_max_f32_dpp %0, %0, %0 row_half_mirror row_mask:0xf bank_mask:0xf\n\t"
        "s_nop 1"
        : "=&v"(r)
        : "v"(x));
    return r;
}

// Where a row's blocks lie: tiles of T x 8 elements, of each `in_tile` blocks of
// 8 or 64 elements; blocks of 64 of 1 << shift tiles (0, or 2 and more) may be
// one.  At most `most` of them.
struct Blocks {
    int log_in_tile, log_units, shift, n;   // blocks of a tile; eights of a block; all blocks
    bool fine;
    __device__ __forceinline__ Blocks(int length, int T, int most) {
        const int tiles = (length + T * 8 - 1) / (T * 8), log_T = 31 - __clz(T);
        fine = tiles <= most / T;
        log_in_tile = fine ? log_T : log_T - 3;
        shift = 0;
        if (!fine && tiles > most >> log_in_tile)
            for (shift = 2; ((tiles - 1) >> shift) + 1 > most >> log_in_tile;) ++shift;
        log_units = (fine ? 0 : 3) + shift;
        n = (((tiles - 1) >> shift) + 1) << log_in_tile;
    }
    // The first element of eight number u of block i, from the part's start; it
    // may lie behind the part's end.
    __device__ __forceinline__ uint32_t element(int i, int u, int T) const {
        const uint32_t tile = (i >> log_in_tile << shift) + (fine ? 0 : u >> 3);
        const uint32_t at = i & ((1 << log_in_tile) - 1);
        return tile * T * 8 + (fine ? at * 8 : at * 64 + (u & 7) * 8);
    }
};

// What a row's sums are once joined: ln S and the entropy.
__device__ __forceinline__ float log_sum(const Soft& x) {
    // +Inf or a NaN is there, or nothing is above -Inf
    return x.m == -INFINITY || !(x.s < INFINITY) ? NAN : log2f(x.s) * kLn2;
}
__device__ __forceinline__ float largest(const Soft& x) {
    return x.s < INFINITY ? x.m : x.s;
}

// A log probability; a distance that passes FP32's range may not after the division.
__device__ __forceinline__ float log_probability(float z, const Soft& x, float tau, float ls) {
    const float d = z - x.m;
    if (__builtin_expect(d == -INFINITY && z > -INFINITY, 0))
        return (float)(((double)z - (double)x.m) / (double)tau - (double)ls);
    return d / tau - ls;
}

// A given token's logit, on its way since the kernel's start.
struct Given {
    bool used;
    float z;
};
template <int FZ>
__device__ __forceinline__ Given load_given(const LogprobArgs& a, int64_t n, const fmt_t<FZ>* z, int i) {
    Given r = {false, 0.0f};
    if (a.logp && i < a.m) {
        const int64_t v = a.idx[n * a.m + i];
        r.used = v >= 0 && v < a.V;
        if (r.used) r.z = fmt_value<FZ>(z[v]);
    }
    return r;
}

// Results of row n but for the top: all threads of the workgroup.
template <int FZ, int T>
__device__ __forceinline__ void row_results(const LogprobArgs& a, int64_t n, const fmt_t<FZ>* z, const Soft& x,
                                            Given first) {
    const float ls = log_sum(x);
    if (threadIdx.x == 0) {
        if (a.stats) {
            a.stats[2 * n] = largest(x);
            a.stats[2 * n + 1] = ls;
        }
        if (a.entropy) a.entropy[n] = ls - kLn2 * (x.t / x.s);
    }
    if (a.logp)
        for (int i = threadIdx.x; i < a.m; i += T) {
            const Given g = i == (int)threadIdx.x ? first : load_given<FZ>(a, n, z, i);
            a.logp[n * a.m + i] = g.used ? log_probability(g.z, x, a.tau, ls) : 0.0f;
        }
}

__device__ __forceinline__ float value_of_order(uint32_t o) {
    return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o);
}

// Place j of row n's top, from its key (0: past the vocabulary's end).
__device__ __forceinline__ void top_result(const LogprobArgs& a, int64_t n, int j, uint64_t key, const Soft& x) {
    const int64_t at = n * a.k + j;
    if (a.top_idx) a.top_idx[at] = key ? index_of(key) : -1;
    if (a.top_logp) {
        const uint32_t o = (uint32_t)(key >> 32);
        const float v = o == 0xFFFFFFFFu ? NAN : value_of_order(o);
        a.top_logp[at] = key ? log_probability(v, x, a.tau, log_sum(x)) : -INFINITY;
    }
}

// The top of a part whose s.count keys that reach the bound are in s.keys, or
// too many for it; written to row n's results or the part's place in the
// workspace.
template <int FZ, int T, bool SPLIT, typename S>
__device__ __forceinline__ void finish_top(const LogprobArgs& a, S& s, int64_t n, const fmt_t<FZ>* z, int v0, int v1,
                                           uint32_t bound, const Soft& x) {
    constexpr int ROOM = S::kRoom;
    const int tid = threadIdx.x;
    __syncthreads();
    int have = s.count;
    if (have > ROOM) {
        // too many: tiles of half the room, the k largest so far in front
        __syncthreads();
        if (tid == 0) s.count = 0;
        __syncthreads();
        for (int w = v0; w < v1; w += ROOM / 2) {
            for (int v = w + tid; v < v1 && v < w + ROOM / 2; v += T) {
                const uint32_t o = order_of(fmt_value<FZ>(z[v]));
                if (o >= bound) s.keys[atomicAdd(&s.count, 1)] = key_of(o, v);
            }
            __syncthreads();
            have = s.count;
            __syncthreads();
            if (have > ROOM / 2 - FP8T_MAX_TOP) {
                const uint64_t* top = top_keys<T>(s, have, a.k);
                have = have < a.k ? have : a.k;
                if (top != s.keys)
                    for (int i = tid; i < have; i += T) s.keys[i] = top[i];
                // what comes later loses against an equal one
                const uint32_t last = have == a.k ? (uint32_t)(top[a.k - 1] >> 32) : 0u;
                if (have == a.k) bound = last == 0xFFFFFFFFu ? last : last + 1;
                if (tid == 0) s.count = have;
                __syncthreads();
            }
        }
        have = s.count;
        __syncthreads();
    }
    const uint64_t* top = top_keys<T>(s, have, a.k);
    for (int j = tid; j < a.k; j += T) {
        const uint64_t key = j < have ? top[j] : 0;
        if (SPLIT) a.part_top[(n * a.parts + blockIdx.z) * a.k + j] = key;
        else top_result(a, n, j, key, x);
    }
}

// The sums of all threads.  red: T / 64 of them, free before the call.
template <int T>
__device__ __forceinline__ Soft block_join(Soft x, Soft* red, float to2) {
    x = wave_join(x, to2);
    if constexpr (T > 64) {
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
        __syncthreads();
        x = red[0];
#pragma unroll
        for (int i = 1; i < T / 64; ++i) x = join(x, red[i], to2);
    }
    return x;
}

// Rows of 2048 elements at most, which no workgroups share: one wave keeps them in
// registers, and nothing is read again.  A group is half the eight elements of a
// load, so that there are as many as alternatives but for the shortest rows, whose
// elements all have room.
constexpr int kShort = 2048;
template <int FZ>
__global__ __launch_bounds__(64) void logprob_short_kernel(LogprobArgs a) {
    constexpr int T = 64, U = kShort / (T * 8), kTile = T * 8, kRoom = 512, kGroups = 2 * T * U;
    __shared__ Selection<kRoom, kGroups> s;
    const int64_t n = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    if (n >= a.N) return;
    const int tid = threadIdx.x;
    const fmt_t<FZ>* z = static_cast<const fmt_t<FZ>*>(a.z) + n * a.z_ld;
    const Consts k(a.to2, Raw<FZ>::kUnit);
    Eight<FZ> e[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (u * kTile < a.V) e[u] = load_logits<FZ>(z, u * kTile + tid * 8, a.V);
    const Given given = load_given<FZ>(a, n, z, tid);
    Soft x = {-INFINITY, 0.0f, 0.0f};
    float top[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float half[2] = {-INFINITY, -INFINITY};
        if (u * kTile < a.V) {                              // the same for all
            float y[1][8], most[1];
            Raw<FZ>::values(e[u], y[0]);
            add_logits<FZ, 1>(x, y, most, k);
#pragma unroll
            for (int h = 0; h < 2; ++h)
                half[h] = max3(fmaxf(y[0][4 * h], y[0][4 * h + 1]), y[0][4 * h + 2], y[0][4 * h + 3]) * Raw<FZ>::kUnit;
        }
        top[u] = fmaxf(half[0], half[1]);
        if (a.k > 0) {
            s.group[u * T + tid] = order_of(half[0]);
            s.group[(U + u) * T + tid] = order_of(half[1]);
        }
    }
    const bool odd = x.s != x.s;                            // a NaN among this thread's
    if (tid == 0) s.count = 0;
    x = block_join<T>(x, nullptr, a.to2);
    row_results<FZ, T>(a, n, z, x, given);
    if (a.k == 0) return;
    const uint32_t bound = find_bound<T>(s, a.k);
    // below every value where there are fewer groups than k (a NaN's bits then)
    const float least = value_of_order(bound);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int v = u * kTile + tid * 8;
        if (v >= a.V || (!odd && top[u] < least)) continue;
        float y[8];
        values8<FZ>(e[u], y);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (!(y[j] < least) && v + j < a.V) {
                const int to = atomicAdd(&s.count, 1);      // the order is made below
                if (to < kRoom) s.keys[to] = key_of(order_of(y[j]), v + j);
            }
    }
    finish_top<FZ, T, false>(a, s, n, z, 0, a.V, bound, x);
}

template <int FZ, int T, bool SPLIT>
__global__ __launch_bounds__(T) void logprob_kernel(LogprobArgs a) {
    constexpr int kBlocks = T < 256 ? T * 8 : T * 4, kRoom = T < 256 ? 512 : T * 4, kGroups = 256;
    __shared__ Selection<kRoom, kGroups> s;
    __shared__ Soft red[T / 64];
    __shared__ float most[kBlocks];
    __shared__ uint16_t chosen[kBlocks];
    __shared__ int reached;
    const int64_t n = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    if (n >= a.N) return;
    const int tid = threadIdx.x, lane = tid & 63;
    const fmt_t<FZ>* z = static_cast<const fmt_t<FZ>*>(a.z) + n * a.z_ld;
    const int v0 = SPLIT ? blockIdx.z * a.per : 0;
    const int v1 = SPLIT && v0 + a.per < a.V ? v0 + a.per : a.V;
    const Consts k(a.to2, Raw<FZ>::kUnit);
    const Given given = SPLIT ? Given{false, 0.0f} : load_given<FZ>(a, n, z, tid);
    Soft x = {-INFINITY, 0.0f, 0.0f};
    constexpr int kAhead = 2, kTile = T * 8;              // kAhead divides four, the least tiles of a block of several
    constexpr float kUnit = Raw<FZ>::kUnit;
    const Blocks blocks(v1 - v0, T, kBlocks);
    const int tiles = (v1 - v0 + kTile - 1) / kTile;
    // the maxima of a batch's or a tile's blocks: whole blocks are written once,
    // those of several tiles by the one lane that has them all
    auto joined = [&](int tile, float top) {
        if (lane & 7) return;
        const int i = (tile >> blocks.shift) * (T / 8) + (tid >> 3);
        most[i] = tile & ((1 << blocks.shift) - 1) ? fmaxf(most[i], top) : top;
    };
    int tile = 0;
    if (v0 + kTile * kAhead <= v1) {
        // whole batches of tiles, the next one on its way
        const fmt_t<FZ>* at = z + v0 + tid * 8;
        Eight<FZ> e[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) e[u] = *reinterpret_cast<const Eight<FZ>*>(at + u * kTile);
        for (; v0 + (tile + kAhead) * kTile <= v1; tile += kAhead) {
            float y[kAhead][8], top[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) Raw<FZ>::values(e[u], y[u]);
            at += kTile * kAhead;
            if (v0 + (tile + 2 * kAhead) * kTile <= v1) {
#pragma unroll
                for (int u = 0; u < kAhead; ++u) e[u] = *reinterpret_cast<const Eight<FZ>*>(at + u * kTile);
            }
            add_logits<FZ, kAhead>(x, y, top, k);
            if (a.k == 0) continue;
            if (blocks.fine) {
#pragma unroll
                for (int u = 0; u < kAhead; ++u) most[(tile + u) * T + tid] = top[u] * kUnit;
            } else if (blocks.shift == 0) {
                // the first lanes of eight write one tile's each
#pragma unroll
                for (int u = 0; u < kAhead; ++u) top[u] = max_of_8_lanes(top[u]);
                const int u = lane & 7;
                float mine = top[0];
#pragma unroll
                for (int i = 1; i < kAhead; ++i) mine = u == i ? top[i] : mine;
                if (u < kAhead) most[(tile + u) * (T / 8) + (tid >> 3)] = mine * kUnit;
            } else {
                float all = top[0];
#pragma unroll
                for (int u = 1; u < kAhead; ++u) all = fmaxf(all, top[u]);
                joined(tile, max_of_8_lanes(all) * kUnit);
            }
        }
    }
    for (; tile < tiles; ++tile) {
        float y[1][8], top[1];
        const int v = v0 + tile * kTile + tid * 8;
        Raw<FZ>::values(load_logits<FZ>(z, v, v1), y[0]);
        add_logits<FZ, 1>(x, y, top, k);
        if (a.k == 0) continue;
        if (blocks.fine) most[tile * T + tid] = top[0] * kUnit;
        else joined(tile, max_of_8_lanes(top[0]) * kUnit);
    }
    if (tid == 0) s.count = reached = 0;
    x = block_join<T>(x, red, a.to2);
    if (!SPLIT) row_results<FZ, T>(a, n, z, x, given);
    else if (tid == 0) a.part_sums[n * a.parts + blockIdx.z] = make_float4(x.m, x.s, x.t, 0.0f);
    if (a.k == 0) return;
    for (int g = tid; g < kGroups; g += T) {
        float top = -INFINITY;
        for (int i = g; i < blocks.n; i += kGroups) top = fmaxf(top, most[i]);
        s.group[g] = order_of(top);
    }
    const uint32_t bound = find_bound<T>(s, a.k);
    // the blocks that reach the bound; all of them where a NaN, which maxima leave out, is about
    const bool odd = x.s != x.s;
    for (int i = tid; i < blocks.n; i += T)
        if (odd || order_of(most[i]) >= bound) chosen[atomicAdd(&reached, 1)] = (uint16_t)i;
    __syncthreads();
    const int items = reached << blocks.log_units;
    // below every value where there are fewer groups than k (a NaN's bits then)
    const float least = value_of_order(bound) * (1.0f / kUnit);   // rounded, it keeps the order
    constexpr int kItems = 4;
    for (int i = tid; i < items; i += T * kItems) {
        Eight<FZ> e[kItems];
        int at[kItems];
#pragma unroll
        for (int u = 0; u < kItems; ++u) {
            const int item = i + u * T, who = item >> blocks.log_units;
            at[u] = v1;
            if (item < items) {
                const uint32_t v = v0 + blocks.element(chosen[who], item - (who << blocks.log_units), T);
                if (v < (uint32_t)v1) at[u] = (int)v;
            }
            if (at[u] < v1) e[u] = load_logits<FZ>(z, at[u], v1);
        }
#pragma unroll
        for (int u = 0; u < kItems; ++u) {
            if (at[u] >= v1) continue;
            float y[8];
            Raw<FZ>::values(e[u], y);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (!(y[j] < least) && at[u] + j < v1) {
                    const int to = atomicAdd(&s.count, 1);  // the order is made below
                    if (to < kRoom) s.keys[to] = key_of(order_of(y[j] * kUnit), at[u] + j);
                }
        }
    }
    finish_top<FZ, T, SPLIT>(a, s, n, z, v0, v1, bound, x);
}

// A row's parts joined: their sums, and the k largest of their tops, which are
// in order: lists are merged two by two, each key's place found by bisection in
// the other list (2 x 128 keys of 32 parts: 7 readings for each of 16 keys of a
// thread, then half as many).
constexpr int kJoinThreads = 256;
template <int FZ>
__global__ __launch_bounds__(kJoinThreads) void logprob_join_kernel(LogprobArgs a) {
    extern __shared__ uint64_t keys[];                      // twice parts x k
    const int64_t n = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    if (n >= a.N) return;
    const int tid = threadIdx.x, k = a.k;
    const fmt_t<FZ>* z = static_cast<const fmt_t<FZ>*>(a.z) + n * a.z_ld;
    const Given given = load_given<FZ>(a, n, z, tid);
    uint64_t *from = keys, *to = keys + a.parts * k;
    for (int i = tid; i < a.parts * k; i += kJoinThreads) from[i] = a.part_top[n * a.parts * k + i];
    const float4* sums = a.part_sums + n * a.parts;
    // every wave joins the parts' sums: lane i has part i's
    const int lane = tid & 63;
    const float4 own = lane < a.parts ? sums[lane] : make_float4(-INFINITY, 0.0f, 0.0f, 0.0f);
    const Soft x = wave_join(Soft{own.x, own.y, own.z}, a.to2);
    row_results<FZ, kJoinThreads>(a, n, z, x, given);
    if (k == 0) return;
    __syncthreads();
    for (int lists = a.parts; lists > 1; lists = (lists + 1) / 2) {
        for (int i = tid; i < lists * k; i += kJoinThreads) {
            const int l = i / k, j = i - l * k, other = l ^ 1;
            const uint64_t mine = from[i];
            int before = 0;                                 // of the other list; an equal one of the first list too
            if (other < lists) {
                const uint64_t* list = from + other * k;
                int lo = 0, hi = k;
                while (lo < hi) {
                    const int mid = (lo + hi) / 2;
                    if (list[mid] > mine || (list[mid] == mine && (l & 1))) lo = mid + 1;
                    else hi = mid;
                }
                before = lo;
            }
            if (j + before < k) to[l / 2 * k + j + before] = mine;
        }
        __syncthreads();
        uint64_t* swap = from;
        from = to;
        to = swap;
    }
    if (tid < k) top_result(a, n, tid, from[tid], x);
}

struct LogprobPlan {
    int parts, per;
    size_t top, bytes;                 // offset of the tops in the workspace; its size
};
LogprobPlan logprob_plan(int64_t N, int64_t V, int64_t k) {
    LogprobPlan p;
    int64_t cus = device_cus();
    if (cus <= 0) cus = 256;
    // parts of 4096 elements at least (the last one may have fewer), as many as fill
    // the chip once
    int64_t parts = N > 0 ? cus / N : 1;
    if (parts > V / 4096) parts = V / 4096;
    if (parts > 32) parts = 32;
    if (parts < 1) parts = 1;
    int64_t per = ((V + parts - 1) / parts + 7) / 8 * 8;
    parts = (V + per - 1) / per;
    p.parts = (int)parts;
    p.per = (int)per;
    p.top = sizeof(float4) * (size_t)N * (size_t)parts;
    p.bytes = parts > 1 ? p.top + sizeof(uint64_t) * (size_t)N * (size_t)parts * (size_t)k : 0;
    return p;
}

dim3 grid_of(int64_t N, int parts) {
    const int64_t across = N < kAcross ? N : kAcross;
    return dim3((unsigned)across, (unsigned)((N + across - 1) / across), (unsigned)parts);
}

template <int FZ, int T>
void launch_rows(const LogprobArgs& a, hipStream_t stream) {
    if (a.parts > 1)
        hipLaunchKernelGGL((logprob_kernel<FZ, T, true>), grid_of(a.N, a.parts), dim3(T), 0, stream, a);
    else
        hipLaunchKernelGGL((logprob_kernel<FZ, T, false>), grid_of(a.N, 1), dim3(T), 0, stream, a);
}
template <int FZ>
void launch(const LogprobArgs& a, hipStream_t stream) {
    // The fewest threads whose sums are not the longer part of a row's time: each
    // row waits for its sums, its bound and its few elements again, and more rows
    // at a time hide that.  FP16, k 20, T 128, 256 and 512, in turn: 8192 x 8192 46,
    // 45 and 69 us; 4096 x 32768 74, 64 and 64 (with k 64 86, 72 and 75); 1024 x
    // 65536 35, 31 and 32; 512 x 131072 61, 35 and 32 (with k 64 75, 43 and 34).
    const int length = a.parts > 1 ? a.per : a.V;
    if (length <= kShort) {
        hipLaunchKernelGGL(logprob_short_kernel<FZ>, grid_of(a.N, 1), dim3(64), 0, stream, a);
    } else if (length <= 8192) {
        launch_rows<FZ, 128>(a, stream);
    } else if (length <= 65536) {
        launch_rows<FZ, 256>(a, stream);
    } else {
        launch_rows<FZ, 512>(a, stream);
    }
    if (a.parts > 1)
        hipLaunchKernelGGL((logprob_join_kernel<FZ>), grid_of(a.N, 1), dim3(kJoinThreads),
                           2 * sizeof(uint64_t) * (size_t)(a.parts * a.k), stream, a);
}

// ---- backward ----------------------------------------------------------------------------

constexpr int kGradThreads = 256;

struct LogprobGradArgs {
    const void* z;
    const int64_t* idx;
    const float* stats;
    const float* entropy;
    const float* d_logp;
    const float* d_entropy;
    void* g;
    int64_t z_ld, g_ld, N;
    int V, m, chunks;                  // chunks of a row
    float tau, to2, scale;             // scale = grad_scale / tau
    bool stream;                       // results past the caches
};

// HBM-bound and without sums over the row: a workgroup owns a chunk of one.  4096
// x 32768 FP16 to FP8: 73 us, 5.5 TB/s; 777 x 50001 floats, three given tokens: 60
// us, 5.2 TB/s (a copy of 1 GiB runs at 5.6).
template <int FZ, int FG>
__global__ __launch_bounds__(kGradThreads) void logprob_bwd_kernel(LogprobGradArgs a) {
    constexpr int kUnits = 4;
    constexpr bool kFours = FZ == FP8T_FMT_F32 || FG == FP8T_FMT_F32;
    extern __shared__ float given[];                        // [m] d_logp, tokens, their logits
    __shared__ float red[kGradThreads / 64];
    int* at = reinterpret_cast<int*>(given + a.m);
    float* logit = given + 2 * a.m;
    const int64_t block = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    const int64_t n = block / a.chunks;
    if (n >= a.N) return;
    const int tid = threadIdx.x;
    const int v0 = (int)(block % a.chunks) * (kGradThreads * 8 * kUnits);
    const int v1 = a.V - v0 > kGradThreads * 8 * kUnits ? v0 + kGradThreads * 8 * kUnits : a.V;
    const fmt_t<FZ>* z = static_cast<const fmt_t<FZ>*>(a.z) + n * a.z_ld;
    fmt_t<FG>* g = static_cast<fmt_t<FG>*>(a.g) + n * a.g_ld;
    Eight<FZ> e[kUnits];
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
        const Cols<kFours> c(u, tid, kGradThreads);
        if (c.any(v1 - v0)) e[u] = load8<FZ>(z + v0, c, v1 - v0);
    }
    const float top = a.stats[2 * n], ls = a.stats[2 * n + 1];
    const float dh = a.d_entropy ? a.d_entropy[n] : 0.0f;
    const float H = a.d_entropy ? a.entropy[n] : 0.0f;
    // the given tokens, their sum, and whether one of them is not 0
    float sum = 0.0f;
    int some = dh != 0.0f;
    if (a.m > 0) {
        for (int i = tid; i < a.m; i += kGradThreads) {
            const int64_t v = a.idx[n * a.m + i];
            const bool used = v >= 0 && v < a.V, here = v >= v0 && v < v1;
            const float d = used ? a.d_logp[n * a.m + i] : 0.0f;
            at[i] = here ? (int)v : -1;
            logit[i] = here ? fmt_value<FZ>(z[v]) : 0.0f;   // before g takes z's place
            given[i] = d;
            sum += d;
            some |= d != 0.0f;
        }
        sum = row_reduce<kGradThreads>(sum, red, RowSum());
        some = __syncthreads_or(some);
    }
    // p (D + dh (l + H)) = 2^d (c1 d + c0), d the distance from the row's largest
    // in base 2: the row's factors are taken once, and no power of a sum
    const float inv = a.scale * exp2f(-ls * kLog2e);
    auto vgpr = [](float x) { return __uint_as_float(in_vgpr(__float_as_uint(x))); };
    const float c0 = vgpr(-inv * (sum + dh * (H - ls))), c1 = vgpr(-inv * dh * kLn2), m = vgpr(top);
    const Consts k(a.to2, Raw<FZ>::kUnit);
    auto gradient = [&](float distance) {
        const float d = distance * k.to2;
        return __builtin_amdgcn_exp2f(d) * __builtin_fmaf(c1, fmaxf(d, kFloor2), c0);
    };
    if (!some) {
        const float none[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            const Cols<kFours> c(u, tid, kGradThreads);
            if (c.any(v1 - v0)) put8<FG>(g + v0, c, v1 - v0, none, a.stream);
        }
        return;
    }
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
        const Cols<kFours> c(u, tid, kGradThreads);
        if (!c.any(v1 - v0)) break;
        float x[8];
        Raw<FZ>::values(e[u], x);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            x[i] = gradient(FZ == FP8T_FMT_F32 ? x[i] - m : __builtin_fmaf(x[i], k.unit, -m));
        put8<FG>(g + v0, c, v1 - v0, x, a.stream);
    }
    if (a.m == 0) return;
    // the given tokens of this chunk, each with the sum of its occurrences, by
    // the first of them -- after the others, above
    __syncthreads();
    for (int i = tid; i < a.m; i += kGradThreads) {
        const int v = at[i];
        if (v < 0) continue;
        float both = 0.0f;
        bool first = true;
        for (int j = 0; j < a.m; ++j)
            if (at[j] == v) {
                first &= j >= i;
                both += given[j];
            }
        if (first) g[v] = fmt_code<FG>(a.scale * both + gradient(logit[i] - top));
    }
}

template <int FZ, int FG>
void launch_bwd(const LogprobGradArgs& a, hipStream_t stream) {
    const int64_t n = a.N * a.chunks, across = n < kAcross ? n : kAcross;
    hipLaunchKernelGGL((logprob_bwd_kernel<FZ, FG>),
                       dim3((unsigned)across, (unsigned)((n + across - 1) / across)), dim3(kGradThreads),
                       3 * sizeof(float) * (size_t)a.m, stream, a);
}

bool logits_ok(const void* z, int z_format, int64_t z_ld, int64_t m, int64_t N, int64_t V, float tau) {
    return N >= 0 && V >= 0 && m >= 0 && m <= kMaxGiven && N <= kMaxGemmDim && V <= kMaxV &&
           float_or_16(z_format) && tau >= 0x1p-30f && tau <= 0x1p30f &&
           (N == 0 || (V > 0 && z && z_ld >= V));
}

}  // namespace
}  // namespace fp8t

using namespace fp8t;

extern "C" size_t token_logprobs_workspace_size(int64_t N, int64_t V, int64_t k) {
    if (N <= 0 || V <= 0 || k < 0 || N > kMaxGemmDim || V > kMaxV || k > FP8T_MAX_TOP) return 0;
    return logprob_plan(N, V, k).bytes;
}

extern "C" int token_logprobs(const void* z, int z_format, int64_t z_ld, const int64_t* idx, int64_t m,
                              int64_t N, int64_t V, float tau, float* logp, float* entropy,
                              float* stats, int64_t k, int64_t* top_idx, float* top_logp,
                              void* workspace, size_t workspace_bytes, hipStream_t stream) {
    if (!logits_ok(z, z_format, z_ld, m, N, V, tau) || k < 0 || k > FP8T_MAX_TOP ||
        (!workspace && workspace_bytes))
        return FP8T_EINVAL;
    if (N == 0) return FP8T_OK;
    if (m == 0) logp = nullptr;
    if (!top_idx && !top_logp) k = 0;
    if (k == 0) top_idx = nullptr, top_logp = nullptr;
    if ((!logp && !entropy && !stats && k == 0) || (logp && !idx)) return FP8T_EINVAL;
    LogprobPlan p = logprob_plan(N, V, k);
    if (workspace_bytes && workspace_bytes < p.bytes) return FP8T_EWORKSPACE;
    if (p.bytes && workspace_bytes && !aligned(workspace, 16)) return FP8T_EINVAL;
    if (p.bytes && !workspace_bytes) p.parts = 1;
    LogprobArgs a;
    a.z = z;
    a.idx = idx;
    a.logp = logp;
    a.entropy = entropy;
    a.stats = stats;
    a.top_idx = top_idx;
    a.top_logp = top_logp;
    a.z_ld = z_ld;
    a.N = N;
    a.V = (int)V;
    a.m = (int)m;
    a.k = (int)k;
    a.parts = p.parts;
    a.per = p.per;
    a.tau = tau;
    a.to2 = kLog2e / tau;
    a.part_sums = static_cast<float4*>(workspace);
    a.part_top = reinterpret_cast<uint64_t*>(static_cast<uint8_t*>(workspace) + (p.parts > 1 ? p.top : 0));
    if (z_format == FP8T_FMT_F32) launch<FP8T_FMT_F32>(a, stream);
    else launch<FP8T_FMT_FP16>(a, stream);
    return launch_status();
}

extern "C" int token_logprobs_bwd(const void* z, int z_format, int64_t z_ld, const int64_t* idx,
                                  int64_t m, const float* stats, const float* entropy,
                                  const float* d_logp, const float* d_entropy, int64_t N, int64_t V,
                                  float tau, float grad_scale, void* g, int g_format, int64_t g_ld,
                                  hipStream_t stream) {
    if (!logits_ok(z, z_format, z_ld, m, N, V, tau) || !storage_format(g_format)) return FP8T_EINVAL;
    if (N == 0) return FP8T_OK;
    if (!stats || !g || g_ld < V || (!d_logp && !d_entropy) || (d_entropy && !entropy) ||
        (d_logp && m > 0 && !idx))
        return FP8T_EINVAL;
    LogprobGradArgs a;
    a.z = z;
    a.idx = idx;
    a.stats = stats;
    a.entropy = entropy;
    a.d_logp = d_logp;
    a.d_entropy = d_entropy;
    a.g = g;
    a.z_ld = z_ld;
    a.g_ld = g_ld;
    a.N = N;
    a.V = (int)V;
    a.m = d_logp ? (int)m : 0;
    a.chunks = (int)((V + kGradThreads * 32 - 1) / (kGradThreads * 32));
    a.tau = tau;
    a.to2 = kLog2e / tau;
    a.scale = grad_scale / tau;
    a.stream = N * V * bytes_of(g_format) > kStreamBytes;
    if (z_format == FP8T_FMT_F32) {
        if (g_format == FP8T_FMT_F32) launch_bwd<FP8T_FMT_F32, FP8T_FMT_F32>(a, stream);
        else if (g_format == FP8T_FMT_FP16) launch_bwd<FP8T_FMT_F32, FP8T_FMT_FP16>(a, stream);
        else launch_bwd<FP8T_FMT_F32, FP8T_FMT_FP8>(a, stream);
    } else {
        if (g_format == FP8T_FMT_F32) launch_bwd<FP8T_FMT_FP16, FP8T_FMT_F32>(a, stream);
        else if (g_format == FP8T_FMT_FP16) launch_bwd<FP8T_FMT_FP16, FP8T_FMT_FP16>(a, stream);
        else launch_bwd<FP8T_FMT_FP16, FP8T_FMT_FP8>(a, stream);
    }
    return launch_status();
}
