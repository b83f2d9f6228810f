// token_logprobs: log probabilities of given tokens, entropy, likeliest tokens.
//
// HBM-bound: a row's logits are read once from memory.  Each thread keeps, of
// its own elements, the largest x, the sum of 2^d and the sum of d 2^d with d
// = (x - largest) log2(e) / tau; the workgroup joins them.  The entropy is
// ln S - (sum of d e^d) / S, both terms of one sign each, so that nothing
// cancels.
//
// The k largest: the threads' maxima, 128 or 256 groups of them, hold at least
// k different elements, so their k-th largest is a bound below which nothing
// can be among the row's k.  Only threads whose own maximum reaches it read
// their elements again (from the caches) and keep what reaches it too; those
// few are ranked by (order of the value, lowest index first).  Where ties or an
// order of the row let more reach it than there is room for, the row is walked
// in tiles, and the bound is raised after each.
//
// Where rows are few, several workgroups share one, each with the k largest of
// its part, and a second kernel joins them.
#include "row_ops.h"

namespace fp8t {
namespace {

constexpr int kMaxGiven = 4096;
constexpr int64_t kAcross = 1 << 20;           // rows along a grid's first dimension
constexpr int64_t kMaxV = INT32_MAX - 16384;   // a thread's positions stay in 32 bits
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

// Largest element, sum of 2^d, sum of d 2^d.
struct Soft {
    float m, s, t;
};
// The sums of x relative to the larger m.
__device__ __forceinline__ void move_to(Soft& x, float m, float to2) {
    if (x.m == m) return;
    const float d = (x.m - m) * to2;                        // negative; -Inf: nothing was there
    const float f = exp2f(d);
    x.t = f > 0.0f ? f * (x.t + d * x.s) : 0.0f * x.s;      // 0, or a NaN kept
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

// The k largest of keys[0, n) to the front, in order; n <= room.  All threads.
template <int T>
__device__ __forceinline__ void top_keys(uint64_t* keys, int n, int k) {
    if (n <= T && n <= 256) {
        // each key's place is the number of larger ones
        const uint64_t mine = (int)threadIdx.x < n ? keys[threadIdx.x] : 0;
        int place = 0;
        if ((int)threadIdx.x < n)
            for (int i = 0; i < n; ++i) place += keys[i] > mine;
        __syncthreads();
        if ((int)threadIdx.x < n && place < k) keys[place] = mine;
        __syncthreads();
        return;
    }
    int size = 2;
    while (size < n) size <<= 1;
    sort_keys<T>(keys, n, size);
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

// What a row's sums are once joined: ln S and the entropy.
__device__ __forceinline__ float log_sum(const Soft& x) {
    // the largest is +Inf, NaN, or nothing was above -Inf
    return x.m == -INFINITY || x.m == INFINITY ? NAN : log2f(x.s) * kLn2;
}

// Results of row n but for the top: all threads of the workgroup.
template <int FZ, int T>
__device__ __forceinline__ void row_results(const LogprobArgs& a, int64_t n, const fmt_t<FZ>* z, Soft x) {
    const float ls = log_sum(x);
    if (threadIdx.x == 0) {
        if (a.stats) {
            a.stats[2 * n] = x.s != x.s ? NAN : x.m;
            a.stats[2 * n + 1] = ls;
        }
        if (a.entropy) a.entropy[n] = ls - kLn2 * (x.t / x.s);
    }
    if (a.logp)
        for (int i = threadIdx.x; i < a.m; i += T) {
            const int64_t v = a.idx[n * a.m + i];
            const bool used = v >= 0 && v < a.V;
            a.logp[n * a.m + i] = used ? (fmt_value<FZ>(z[v]) - x.m) / a.tau - ls : 0.0f;
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
        a.top_logp[at] = key ? (v - x.m) / a.tau - log_sum(x) : -INFINITY;
    }
}

template <int FZ, int T, bool SPLIT>
__global__ __launch_bounds__(T) void logprob_kernel(LogprobArgs a) {
    constexpr int kRoom = T * 8, kWaves = T / 64, kGroups = 256;
    __shared__ uint64_t keys[kRoom];
    __shared__ Soft red[kWaves];
    __shared__ uint32_t group[kGroups];
    __shared__ uint32_t bound_of;
    __shared__ int count;
    const int64_t n = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    if (n >= a.N) return;
    const int tid = threadIdx.x, lane = tid & 63;
    const fmt_t<FZ>* z = static_cast<const fmt_t<FZ>*>(a.z) + n * a.z_ld;
    const int v0 = SPLIT ? blockIdx.z * a.per : 0;
    const int v1 = SPLIT && v0 + a.per < a.V ? v0 + a.per : a.V;
    const float to2 = a.to2;
    Soft x = {-INFINITY, 0.0f, 0.0f};
    constexpr int kAhead = 4;
    for (int v = v0 + tid * 8; v < v1; v += T * 8 * kAhead) {
        Eight<FZ> e[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (v + u * T * 8 < v1) e[u] = load_logits<FZ>(z, v + u * T * 8, v1);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (v + u * T * 8 >= v1) break;
            float y[8];
            values8<FZ>(e[u], y);
            float top = y[0];
#pragma unroll
            for (int i = 1; i < 8; ++i) top = fmaxf(top, y[i]);
            if (top > x.m) move_to(x, top, to2);
            const float m = x.m == -INFINITY ? 0.0f : x.m;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = (y[i] - m) * to2, p = __builtin_amdgcn_exp2f(d);
                x.s += p;
                x.t += fmaxf(d, -160.0f) * p;               // d = -Inf adds 0
            }
        }
    }
    const float own = x.m;
    const bool odd = x.s != x.s;                            // a NaN, or +Inf, among this thread's
#pragma unroll
    for (int d = 32; d; d >>= 1) {
        Soft y = {__shfl_xor(x.m, d), __shfl_xor(x.s, d), __shfl_xor(x.t, d)};
        x = join(x, y, to2);
    }
    if (lane == 0) red[tid >> 6] = x;
    if (a.k > 0) {
        if (tid == 0) count = 0;
        // the threads' maxima in groups of T / 256 neighbours
        uint32_t o = order_of(own);                         // a NaN beside it is above
#pragma unroll
        for (int d = 1; d < T / kGroups; d <<= 1) o = max(o, (uint32_t)__shfl_xor((int)o, d));
        if (tid % (T / kGroups) == 0) group[tid / (T / kGroups)] = o;
    }
    __syncthreads();
    x = red[0];
#pragma unroll
    for (int i = 1; i < kWaves; ++i) x = join(x, red[i], to2);
    if (!SPLIT) row_results<FZ, T>(a, n, z, x);
    else if (tid == 0) a.part_sums[n * a.parts + blockIdx.z] = make_float4(x.m, x.s, x.t, 0.0f);
    if (a.k == 0) return;
    if (tid < 64) {
        // a bound that k groups at least reach: its bits from the highest on
        uint32_t g[kGroups / 64], bound = 0;
#pragma unroll
        for (int i = 0; i < kGroups / 64; ++i) g[i] = group[i * 64 + lane];
        for (int b = 31; b >= 0; --b) {
            const uint32_t tried = bound | (1u << b);
            int reach = 0;
#pragma unroll
            for (int i = 0; i < kGroups / 64; ++i) reach += __popcll(__ballot(g[i] >= tried));
            if (reach >= a.k) bound = tried;
            if (reach == a.k) break;
        }
        if (lane == 0) bound_of = bound;
    }
    __syncthreads();
    uint32_t bound = bound_of;
    // elements that reach the bound, of threads whose largest does
    if (odd || order_of(own) >= bound) {
        for (int v = v0 + tid * 8; v < v1; v += T * 8) {
            float y[8];
            values8<FZ>(load_logits<FZ>(z, v, v1), y);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t o = order_of(y[i]);
                if (o >= bound && v + i < v1) {
                    const int at = atomicAdd(&count, 1);    // the order is made below
                    if (at < kRoom) keys[at] = key_of(o, v + i);
                }
            }
        }
    }
    __syncthreads();
    int have = count;
    if (have > kRoom) {
        // too many: tiles of half the room, the k largest so far in front
        __syncthreads();
        if (tid == 0) count = 0;
        __syncthreads();
        for (int w = v0; w < v1; w += kRoom / 2) {
            const int v = w + tid * 4;
            for (int i = 0; i < 4; ++i) {
                if (v + i >= v1) break;
                const uint32_t o = order_of(fmt_value<FZ>(z[v + i]));
                if (o >= bound) {
                    const int at = atomicAdd(&count, 1);
                    keys[at] = key_of(o, v + i);
                }
            }
            __syncthreads();
            have = count;
            __syncthreads();
            if (have > kRoom / 2 - FP8T_MAX_TOP) {
                top_keys<T>(keys, have, a.k);
                have = have < a.k ? have : a.k;
                // what comes later loses against an equal one
                const uint32_t last = have == a.k ? (uint32_t)(keys[a.k - 1] >> 32) : 0u;
                if (have == a.k) bound = last == 0xFFFFFFFFu ? last : last + 1;
                if (tid == 0) count = have;
                __syncthreads();
            }
        }
        have = count;
        __syncthreads();
    }
    top_keys<T>(keys, have, a.k);
    if (tid < a.k) {
        const uint64_t key = tid < have ? keys[tid] : 0;
        if (SPLIT) a.part_top[(n * a.parts + blockIdx.z) * a.k + tid] = key;
        else top_result(a, n, tid, key, x);
    }
}

// A row's parts joined: their sums, and the k largest of their tops.
constexpr int kJoinThreads = 256;
template <int FZ>
__global__ __launch_bounds__(kJoinThreads) void logprob_join_kernel(LogprobArgs a) {
    extern __shared__ uint64_t keys[];                      // parts x k, up to a power of two
    const int64_t n = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    if (n >= a.N) return;
    const int tid = threadIdx.x;
    const float4* sums = a.part_sums + n * a.parts;
    Soft x = {sums[0].x, sums[0].y, sums[0].z};
    for (int i = 1; i < a.parts; ++i) x = join(x, Soft{sums[i].x, sums[i].y, sums[i].z}, a.to2);
    row_results<FZ, kJoinThreads>(a, n, static_cast<const fmt_t<FZ>*>(a.z) + n * a.z_ld, x);
    if (a.k == 0) return;
    const int all = a.parts * a.k;
    for (int i = tid; i < all; i += kJoinThreads) keys[i] = a.part_top[n * all + i];
    __syncthreads();
    top_keys<kJoinThreads>(keys, all, a.k);
    if (tid < a.k) top_result(a, n, tid, keys[tid], x);
}

struct LogprobPlan {
    int threads, parts, per;
    size_t top, bytes;                 // offset of the tops in the workspace; its size
};
LogprobPlan logprob_plan(int64_t N, int64_t V, int64_t k) {
    LogprobPlan p;
    int64_t cus = device_cus();
    if (cus <= 0) cus = 256;
    // parts of 4096 elements at least, as many as fill the chip once
    int64_t parts = N > 0 ? cus / N : 1;
    if (parts > V / 4096) parts = V / 4096;
    if (parts > 32) parts = 32;
    if (parts < 1) parts = 1;
    int64_t per = ((V + parts - 1) / parts + 7) / 8 * 8;
    parts = (V + per - 1) / per;
    p.parts = (int)parts;
    p.per = (int)per;
    p.threads = per <= 16384 ? 256 : per <= 65536 ? 512 : 1024;
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
void launch(const LogprobArgs& a, int threads, hipStream_t stream) {
    if (threads == 256) launch_rows<FZ, 256>(a, stream);
    else if (threads == 512) launch_rows<FZ, 512>(a, stream);
    else launch_rows<FZ, 1024>(a, stream);
    if (a.parts > 1) {
        int size = 2;
        while (size < a.parts * a.k) size <<= 1;
        hipLaunchKernelGGL((logprob_join_kernel<FZ>), grid_of(a.N, 1), dim3(kJoinThreads),
                           sizeof(uint64_t) * (size_t)size, stream, a);
    }
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
};

// HBM-bound and without sums over the row: a workgroup owns a chunk of one.
template <int FZ, int FG>
__global__ __launch_bounds__(kGradThreads) void logprob_bwd_kernel(LogprobGradArgs a) {
    constexpr int kUnits = 4;
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
        const int v = v0 + (u * kGradThreads + tid) * 8;
        if (v < v1) e[u] = load_logits<FZ>(z, v, v1);
    }
    const float top = a.stats[2 * n], ls2 = a.stats[2 * n + 1] * kLog2e;
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
    auto gradient = [&](float x, float both) {
        // the exponent is that of the distance from the row's largest, base 2
        const float l = (x - top) * a.to2 - ls2, p = __builtin_amdgcn_exp2f(l);
        const float f = sum + dh * (fmaxf(l, -160.0f) * kLn2 + H);
        return a.scale * (both - p * f);
    };
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
        const int v = v0 + (u * kGradThreads + tid) * 8;
        if (v >= v1) break;
        float x[8];
        values8<FZ>(e[u], x);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = some ? gradient(x[i], 0.0f) : 0.0f;
        store_some<FG>(g + v, left8(v, v1), x);
    }
    if (a.m == 0 || !some) return;
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
        if (first) g[v] = fmt_code<FG>(gradient(logit[i], both));
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
    if (p.bytes && !workspace_bytes) {
        p.parts = 1;
        p.threads = 1024;
    }
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
    if (z_format == FP8T_FMT_F32) launch<FP8T_FMT_F32>(a, p.threads, stream);
    else launch<FP8T_FMT_FP16>(a, p.threads, stream);
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
