// embed_fwd, embed_bwd: rows of a table by tokens, and the table's gradient.
//
// Forward: HBM-bound, one pass.  A thread owns eight columns of four rows,
// whose tokens and table rows are loaded together.  16384 tokens of a text's
// frequencies, 50001 x 2048 FP16 to floats: 26 us, 6.1 TB/s (a copy of 1 GiB runs
// at 5.6, a fill at 6.9).  One, two or eight rows change that by 3%.
//
// Backward: the tokens are sorted, so that every row of the gradient is summed
// by one reader of its errors and written once, with no atomics.  Two or three
// launches:
//   index  -- workgroup r owns R rows of the vocabulary and reads all tokens
//             twice: first it counts each row's tokens per wave and those below
//             its rows (that is where its part of the sorted list begins), then
//             every wave places its own tokens in order.  No sorting passes, no
//             scan over workgroups: reading 16384 tokens in each of 256
//             workgroups is 32 MB from the L2s, 8 us.  A wave that meets more than
//             kSeen of its rows' tokens reads its share again, which the frequent
//             tokens of a text bring about from some 50000 on: 65536 tokens 64
//             us (the sums of 512 columns 31, of 2048 133), 262144 238 us, 2^20
//             936 us, what such calls take longest for.
//   sum    -- a workgroup takes a piece of the sorted tokens, each of its groups
//             of lanes the runs (equal tokens) that begin in its share.  The
//             errors of eight tokens are on their way whatever runs they belong
//             to (run by run: 107 us where this takes 33).  A run of more than
//             kLong is cut at the shares' borders: the parts' sums meet in LDS,
//             in order, and those of runs that leave the piece go to the
//             workspace.  Sums are doubles (a frequent token's errors cancel; the
//             vector ALUs are idle).  Other workgroups write the rows that no
//             token names.
//   join   -- adds the parts of such runs in their order.
// 16384 tokens into 32768 x 1024 floats: 8 + 33 + 5 us; the gradient's 134 MB and
// the errors' 34 are 30 us of a copy's rate.
#include "row_ops.h"

namespace fp8t {
namespace {

constexpr int kThreads = 256;
constexpr int64_t kAcross = 1 << 20;   // workgroups along a grid's first dimension

struct EmbedArgs {
    const int64_t* tokens;
    const void* table;
    void* y;
    int64_t T, V, W, t_ld, y_ld;
    float scale;
    int log_lanes;                     // lanes of a row: 1 << log_lanes, each with eight columns at a time
    bool stream;                       // results past the caches
};

template <int FT, int FY>
__global__ __launch_bounds__(kThreads) void embed_kernel(EmbedArgs a) {
    constexpr int kRows = 4;
    constexpr bool kFours = FT == FP8T_FMT_F32 || FY == FP8T_FMT_F32;
    const int lanes = 1 << a.log_lanes, per = kThreads >> a.log_lanes, lane = threadIdx.x & (lanes - 1);
    const int64_t step = (int64_t)gridDim.x * per * kRows;
    for (int64_t t0 = (int64_t)blockIdx.x * per * kRows + (threadIdx.x >> a.log_lanes); t0 < a.T; t0 += step) {
        int64_t tok[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const int64_t t = t0 + r * per;
            tok[r] = t < a.T ? a.tokens[t] : -1;
        }
        for (int64_t u = 0; u * 8 * lanes < a.W; ++u) {
            const Cols<kFours> c(u, lane, lanes);
            if (!c.any(a.W)) break;
            Eight<FT> e[kRows] = {};
#pragma unroll
            for (int r = 0; r < kRows; ++r)
                if ((uint64_t)tok[r] < (uint64_t)a.V)
                    e[r] = load8<FT>(static_cast<const fmt_t<FT>*>(a.table) + tok[r] * a.t_ld, c, a.W);
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                const int64_t t = t0 + r * per;
                if (t >= a.T) break;
                float x[8];
                values8<FT>(e[r], x);
                const bool used = (uint64_t)tok[r] < (uint64_t)a.V;
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = used ? x[i] * a.scale : 0.0f;
                put8<FY>(static_cast<fmt_t<FY>*>(a.y) + t * a.y_ld, c, a.W, x, a.stream);
            }
        }
    }
}

// Lanes (a power of two up to `most`) that hold a row's units of eight.
int log_lanes(int64_t W, int most) {
    int l = 0;
    while ((1 << l) < most && (int64_t)(8 << l) < W) ++l;
    return l;
}

template <int FT, int FY>
void launch_fwd(const EmbedArgs& a, hipStream_t stream) {
    const int64_t per = 4 * (kThreads >> a.log_lanes), n = (a.T + per - 1) / per;
    hipLaunchKernelGGL((embed_kernel<FT, FY>), dim3((unsigned)(n < kAcross ? n : kAcross)), dim3(kThreads), 0,
                       stream, a);
}

// ---- backward ----------------------------------------------------------------------------

constexpr int kIndexThreads = 1024, kWaves = kIndexThreads / 64, kMaxRows = 512;
constexpr int kSeen = 192;             // tokens of its rows that a wave of the index kernel keeps
constexpr int kMinShare = 4, kShare = 16;   // sorted tokens of a group of lanes
constexpr int kLong = 32;              // the longest run that is not cut
constexpr int kZeroRows = 16;          // rows that a wave looks at for those without a token
static_assert(kLong >= kShare, "a run longer than kLong passes a border of its share");

struct GradArgs {
    const int64_t* tokens;
    const void* e;
    void* g;
    int64_t T, V, W, e_ld, g_ld;
    float scale;
    int R;                             // vocabulary rows per index workgroup
    int log_lanes;                     // lanes of a row of errors, eight columns each
    int slabs;                         // column slabs of 8 << log_lanes
    int log_columns, join_slabs;       // columns of a group of threads of the join, its column slabs
    int share, piece;                  // sorted tokens of a group of lanes, of a workgroup
    int64_t pieces, piece_blocks, zero_blocks;
    int* start;                        // V + 1: a row's first sorted token
    int2* list;                        // T: (token, position), sorted
    double* parts;                     // pieces x 2 x W: sums of cut runs
    bool stream;                       // results past the caches
};

__global__ __launch_bounds__(kIndexThreads) void embed_index_kernel(GradArgs a) {
    extern __shared__ int hist[];                           // kWaves x R
    __shared__ int2 seen[kWaves][kSeen];
    __shared__ int red[kWaves];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const uint64_t below_me = (1ull << lane) - 1;
    for (int i = tid; i < kWaves * a.R; i += kIndexThreads) hist[i] = 0;
    __syncthreads();
    const int64_t v0 = (int64_t)blockIdx.x * a.R;
    const int rows = (int)(a.V - v0 < a.R ? a.V - v0 : a.R);
    // this wave's tokens: whole groups of 64
    const int64_t share = ((a.T + 63) / 64 + kWaves - 1) / kWaves * 64;
    const int64_t i0 = wave * share, i1 = i0 + share < a.T ? i0 + share : a.T;
    int* mine = hist + wave * a.R;
    int below = 0, n = 0;                                   // n: of this wave's rows so far
    constexpr int kAhead = 8;
    for (int64_t i = i0; i < i1; i += 64 * kAhead) {
        int64_t tok[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int64_t at = i + 64 * u + lane;
            tok[u] = at < i1 ? a.tokens[at] : -1;
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            below += tok[u] >= 0 && tok[u] < v0;
            const bool in = tok[u] >= v0 && tok[u] < v0 + rows;
            const uint64_t m = __ballot(in);
            if (m == 0) continue;
            if (in) {
                const int id = (int)(tok[u] - v0), at = n + __popcll(m & below_me);
                atomicAdd(mine + id, 1);                    // of one wave: no order to it
                if (at < kSeen) seen[wave][at] = make_int2(id, (int)(i + 64 * u + lane));
            }
            n += __popcll(m);
        }
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) below += __shfl_xor(below, d);
    if (lane == 0) red[wave] = below;
    __syncthreads();
    int base = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) base += red[w];
    __syncthreads();
    // where each wave's tokens of each row begin: thread r sums row r over the
    // waves, the rows are scanned over the workgroup (R <= kIndexThreads)
    int sum = 0;
    if (tid < rows)
        for (int w = 0; w < kWaves; ++w) sum += hist[w * a.R + tid];
    int scan = sum;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int up = __shfl_up(scan, d);
        if (lane >= d) scan += up;
    }
    if (lane == 63) red[wave] = scan;
    __syncthreads();
    for (int w = 0; w < wave; ++w) scan += red[w];
    if (tid < rows) {
        int at = base + scan - sum;
        a.start[v0 + tid] = at;
        for (int w = 0; w < kWaves; ++w) {
            const int c = hist[w * a.R + tid];
            hist[w * a.R + tid] = at;
            at += c;
        }
        if (v0 + tid == a.V - 1) a.start[a.V] = at;
    }
    __syncthreads();
    // a group of this wave's tokens in their order: equal ones take consecutive
    // places, found by comparing the bits of all lanes at once
    auto place = [&](bool in, int id, int pos) {
        uint64_t same = __ballot(in);
        if (same == 0) return;
        for (int b = 0; (a.R - 1) >> b; ++b) {
            const uint64_t set = __ballot((id >> b) & 1);
            same &= (id >> b) & 1 ? set : ~set;
        }
        const int first = in ? __ffsll((unsigned long long)same) - 1 : lane;
        int at = 0;
        if (in && lane == first) at = atomicAdd(mine + id, __popcll(same));
        at = __shfl(at, first) + __popcll(same & below_me);
        if (in) a.list[at] = make_int2((int)(v0 + id), pos);
    };
    if (n <= kSeen) {
        for (int i = 0; i < n; i += 64) {
            const bool in = i + lane < n;
            const int2 s = in ? seen[wave][i + lane] : make_int2(0, 0);
            place(in, s.x, s.y);
        }
        return;
    }
    for (int64_t i = i0; i < i1; i += 64 * kAhead) {
        int64_t tok[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int64_t at = i + 64 * u + lane;
            tok[u] = at < i1 ? a.tokens[at] : -1;
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            place(tok[u] >= v0 && tok[u] < v0 + rows, (int)(tok[u] - v0), (int)(i + 64 * u + lane));
    }
}

template <int FG, bool FOURS>
__device__ __forceinline__ void grad_out(const GradArgs& a, int64_t v, const Cols<FOURS>& c, const double* sum) {
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = (float)(sum[i] * (double)a.scale);
    put8<FG>(static_cast<fmt_t<FG>*>(a.g) + v * a.g_ld, c, a.W, y, a.stream);
}

// A cut run's part, in the workspace.
template <bool FOURS>
__device__ __forceinline__ void put_sums(const GradArgs& a, int64_t part, const Cols<FOURS>& c, const double* sum) {
    double* to = a.parts + part * a.W;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (c.has(i, a.W)) to[i < 4 ? c.a + i : c.b + i - 4] = sum[i];
}

template <int FE, int FG>
__global__ __launch_bounds__(kThreads) void embed_sum_kernel(GradArgs a) {
    constexpr bool kFours = FE == FP8T_FMT_F32 || FG == FP8T_FMT_F32;
    const int64_t block = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    if (block >= a.piece_blocks) {
        // rows without a token: among kZeroRows a wave
        const int64_t z = block - a.piece_blocks;
        const int lane = threadIdx.x & 63;
        const int64_t v0 = (z * (kThreads / 64) + (threadIdx.x >> 6)) * kZeroRows, v = v0 + lane;
        const bool none = lane < kZeroRows && v < a.V && a.start[v] == a.start[v + 1];
        uint64_t todo = __ballot(none);
        const float zero[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        while (todo) {
            const int64_t at = v0 + __ffsll((unsigned long long)todo) - 1;
            todo &= todo - 1;
            for (int64_t u = 0; u * 512 < a.W; ++u) {
                const Cols<kFours> c(u, lane, 64);
                if (c.any(a.W)) put8<FG>(static_cast<fmt_t<FG>*>(a.g) + at * a.g_ld, c, a.W, zero, a.stream);
            }
        }
        return;
    }
    const int per = kThreads >> a.log_lanes, group = threadIdx.x >> a.log_lanes;
    const int lane = threadIdx.x & ((1 << a.log_lanes) - 1);
    const int64_t p = block / a.slabs;
    const Cols<kFours> c(block % a.slabs, lane, 1 << a.log_lanes);
    const int n = a.start[a.V];
    if (p * a.piece >= n) return;
    // what a group leaves of cut runs: [0] of one that began before its share,
    // [1] of one that begins there: eight sums of each thread
    __shared__ double2 part[2][4][kThreads];
    __shared__ int left[2][kThreads];                       // their tokens, -1: none
    const int from = (int)p * a.piece + group * a.share, to = from + a.share < n ? from + a.share : n;
    if (lane == 0) left[0][group] = left[1][group] = -1;
    if (from < n) {
        const fmt_t<FE>* e = static_cast<const fmt_t<FE>*>(a.e);
        const bool mine = c.any(a.W);                       // not past the row's end
        const int head = a.list[from].x, tail = a.list[to - 1].x;
        const int head_begin = a.start[head], head_end = a.start[head + 1];
        const int tail_begin = a.start[tail], tail_end = a.start[tail + 1];
        int i = from, last = to;
        const bool cut_head = head_begin < from && head_end - head_begin > kLong;
        const bool cut_tail = tail_begin >= from && tail_end - tail_begin > kLong;
        if (head_begin < from && !cut_head) i = head_end;   // the share where it began sums it
        if (tail_begin >= i && !cut_tail && tail_end > to) last = tail_end;
        if (lane == 0 && cut_head) left[0][group] = head;
        if (lane == 0 && cut_tail) left[1][group] = tail;
        double sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        int v = i < last ? a.list[i].x : -1;
        auto flush = [&]() {
            if ((v == head && cut_head) || (v == tail && cut_tail)) {
                const int at = v == head && cut_head ? 0 : 1;
#pragma unroll
                for (int k = 0; k < 4; ++k) part[at][k][threadIdx.x] = make_double2(sum[2 * k], sum[2 * k + 1]);
            } else if (mine) {
                grad_out<FG>(a, v, c, sum);
            }
        };
        constexpr int kAhead = 8;
        int2 next[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) next[u] = a.list[i + u < last ? i + u : from];
        for (int j = i; j < last; j += kAhead) {
            Eight<FE> x[kAhead] = {};
            int tok[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                tok[u] = next[u].x;
                if (j + u < last && mine) x[u] = load8<FE>(e + (int64_t)next[u].y * a.e_ld, c, a.W);
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                next[u] = a.list[j + kAhead + u < last ? j + kAhead + u : from];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (j + u >= last) break;
                if (tok[u] != v) {
                    flush();
                    v = tok[u];
#pragma unroll
                    for (int k = 0; k < 8; ++k) sum[k] = 0.0;
                }
                float w[8];
                values8<FE>(x[u], w);
#pragma unroll
                for (int k = 0; k < 8; ++k) sum[k] += (double)w[k];
            }
        }
        if (i < last) flush();
    }
    __syncthreads();
    // the first group joins the parts of cut runs in their order; a run that
    // began before the piece or goes on behind it leaves a part of its own
    if (group > 0 || !c.any(a.W)) return;
    double sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    int v = -1;
    bool inside = false;                                    // the run began in this piece
    auto done = [&](bool more) {
        if (v < 0) return;
        if (inside && !more) grad_out<FG>(a, v, c, sum);
        else put_sums(a, p * 2 + inside, c, sum);
    };
    for (int g = 0; g < per; ++g)
#pragma unroll
        for (int at = 0; at < 2; ++at) {
            if (left[at][g] < 0) continue;
            if (left[at][g] != v) {
                done(false);
                v = left[at][g];
                inside = at == 1;
#pragma unroll
                for (int k = 0; k < 8; ++k) sum[k] = 0.0;
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const double2 x = part[at][k][(g << a.log_lanes) + lane];
                sum[2 * k] += x.x;
                sum[2 * k + 1] += x.y;
            }
        }
    done(v >= 0 && a.start[v + 1] > (p + 1) * a.piece);
}

// The cut run that begins in piece p and goes on behind it, if one does: a thread
// owns a column.
template <int FG>
__global__ __launch_bounds__(kThreads) void embed_join_kernel(GradArgs a) {
    const int64_t block = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    const int64_t p = block / a.join_slabs * (kThreads >> a.log_columns) + (threadIdx.x >> a.log_columns);
    const int64_t c = (block % a.join_slabs << a.log_columns) + (threadIdx.x & ((1 << a.log_columns) - 1));
    const int n = a.start[a.V];
    if ((p + 1) * a.piece >= n || c >= a.W) return;
    const int v = a.list[(p + 1) * a.piece - 1].x, begin = a.start[v], end = a.start[v + 1];
    if (begin < p * a.piece || end <= (p + 1) * a.piece || end - begin <= kLong) return;
    const int64_t last = (end - 1) / a.piece;
    double sum = a.parts[(p * 2 + 1) * a.W + c];
    constexpr int kAhead = 16;
    for (int64_t q = p + 1; q <= last; q += kAhead) {
        double x[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) x[u] = q + u <= last ? a.parts[(q + u) * 2 * a.W + c] : 0.0;
#pragma unroll
        for (int u = 0; u < kAhead; ++u) sum += x[u];
    }
    static_cast<fmt_t<FG>*>(a.g)[v * a.g_ld + c] = fmt_code<FG>((float)(sum * (double)a.scale));
}

struct GradPlan {
    int R, log_lanes, slabs, share, piece;
    int64_t pieces;
    size_t list, parts, bytes;         // offsets into the workspace: start, list, parts
};

GradPlan grad_plan(int64_t T, int64_t V, int64_t W) {
    GradPlan p;
    const int64_t r = (V + 255) / 256;
    p.R = (int)(r < 16 ? 16 : r > kMaxRows ? kMaxRows : r);
    p.log_lanes = log_lanes(W, 64);
    p.slabs = (int)((W + (8 << p.log_lanes) - 1) / (8 << p.log_lanes));
    // small shares where few tokens would leave CUs idle: 257 tokens of 256 columns
    // 13 us with 16, 10 with 4
    const int64_t waves = (T * p.slabs << p.log_lanes) / 64;   // of one token each
    p.share = (int)(waves / 2048 < kMinShare ? kMinShare : waves / 2048 > kShare ? kShare : waves / 2048);
    p.piece = p.share * (kThreads >> p.log_lanes);
    p.pieces = (T + p.piece - 1) / p.piece;
    auto up = [](size_t n) { return (n + 15) & ~(size_t)15; };
    p.list = up(sizeof(int) * (size_t)(V + 1));
    p.parts = p.list + up(sizeof(int2) * (size_t)T);
    p.bytes = p.parts + (p.pieces > 1 ? sizeof(double) * 2 * (size_t)W * (size_t)p.pieces : 0);
    return p;
}

dim3 grid_of(int64_t n) {
    const int64_t across = n < kAcross ? n : kAcross;
    return dim3((unsigned)across, (unsigned)((n + across - 1) / across));
}

template <int FE, int FG>
void launch_bwd(GradArgs a, hipStream_t stream) {
    const size_t lds = sizeof(int) * kWaves * (size_t)a.R;
    hipLaunchKernelGGL(embed_index_kernel, dim3((unsigned)((a.V + a.R - 1) / a.R)), dim3(kIndexThreads), lds,
                       stream, a);
    a.piece_blocks = a.pieces * a.slabs;
    a.zero_blocks = (a.V + kThreads / 64 * kZeroRows - 1) / (kThreads / 64 * kZeroRows);
    hipLaunchKernelGGL((embed_sum_kernel<FE, FG>), grid_of(a.piece_blocks + a.zero_blocks), dim3(kThreads), 0, stream, a);
    if (a.pieces > 1) {
        a.log_columns = 0;
        while ((1 << a.log_columns) < kThreads && (1 << a.log_columns) < a.W) ++a.log_columns;
        a.join_slabs = (int)((a.W + (1 << a.log_columns) - 1) >> a.log_columns);
        const int64_t per = kThreads >> a.log_columns;
        hipLaunchKernelGGL((embed_join_kernel<FG>), grid_of((a.pieces + per - 1) / per * a.join_slabs),
                           dim3(kThreads), 0, stream, a);
    }
}

bool grad_sizes_ok(int64_t T, int64_t V, int64_t W) {
    return T >= 0 && V >= 0 && W >= 0 && T <= kMaxGemmDim && W <= kMaxGemmDim && V <= FP8T_MAX_VOCAB;
}

// fn<FX, FY>(a, stream) for formats known at run time.
#define FP8T_BY_FORMATS(fn, fx, fy, ...)                                                       \
    switch ((fx) * 3 + (fy)) {                                                                 \
        case 0: fn<FP8T_FMT_F32, FP8T_FMT_F32>(__VA_ARGS__); break;                            \
        case 1: fn<FP8T_FMT_F32, FP8T_FMT_FP16>(__VA_ARGS__); break;                           \
        case 2: fn<FP8T_FMT_F32, FP8T_FMT_FP8>(__VA_ARGS__); break;                            \
        case 3: fn<FP8T_FMT_FP16, FP8T_FMT_F32>(__VA_ARGS__); break;                           \
        case 4: fn<FP8T_FMT_FP16, FP8T_FMT_FP16>(__VA_ARGS__); break;                          \
        case 5: fn<FP8T_FMT_FP16, FP8T_FMT_FP8>(__VA_ARGS__); break;                           \
        case 6: fn<FP8T_FMT_FP8, FP8T_FMT_F32>(__VA_ARGS__); break;                            \
        case 7: fn<FP8T_FMT_FP8, FP8T_FMT_FP16>(__VA_ARGS__); break;                           \
        default: fn<FP8T_FMT_FP8, FP8T_FMT_FP8>(__VA_ARGS__); break;                           \
    }

}  // namespace
}  // namespace fp8t

using namespace fp8t;

extern "C" int embed_fwd(const int64_t* tokens, int64_t T, const void* table, int table_format,
                         int64_t table_ld, int64_t V, int64_t W, float scale, void* y, int y_format,
                         int64_t y_ld, hipStream_t stream) {
    if (T < 0 || V < 0 || W < 0 || T > kMaxGemmDim || V > kMaxGemmDim || W > kMaxGemmDim ||
        !storage_format(table_format) || !storage_format(y_format))
        return FP8T_EINVAL;
    if (T == 0 || W == 0) return FP8T_OK;
    if (!tokens || !matrix_ok(table, table_ld, V, W) || !matrix_ok(y, y_ld, T, W)) return FP8T_EINVAL;
    EmbedArgs a;
    a.tokens = tokens;
    a.table = table;
    a.y = y;
    a.T = T;
    a.V = V;
    a.W = W;
    a.t_ld = table_ld;
    a.y_ld = y_ld;
    a.scale = scale;
    a.log_lanes = log_lanes(W, kThreads);
    a.stream = T * W * bytes_of(y_format) > kStreamBytes;
    FP8T_BY_FORMATS(launch_fwd, table_format, y_format, a, stream)
    return launch_status();
}

extern "C" size_t embed_bwd_workspace_size(int64_t T, int64_t V, int64_t W) {
    if (!grad_sizes_ok(T, V, W) || V == 0 || W == 0) return 0;
    return grad_plan(T, V, W).bytes;
}

extern "C" int embed_bwd(const int64_t* tokens, int64_t T, const void* e, int e_format, int64_t e_ld,
                         int64_t V, int64_t W, float scale, void* g, int g_format, int64_t g_ld,
                         void* workspace, size_t workspace_bytes, hipStream_t stream) {
    if (!grad_sizes_ok(T, V, W) || !storage_format(e_format) || !storage_format(g_format) ||
        (!workspace && workspace_bytes))
        return FP8T_EINVAL;
    if (V == 0 || W == 0) return FP8T_OK;
    if ((T > 0 && !tokens) || !matrix_ok(e, e_ld, T, W) || !matrix_ok(g, g_ld, V, W) ||
        !aligned(workspace, 16))
        return FP8T_EINVAL;
    const GradPlan p = grad_plan(T, V, W);
    if (workspace_bytes < p.bytes) return FP8T_EWORKSPACE;
    GradArgs a = {};
    a.tokens = tokens;
    a.e = e;
    a.g = g;
    a.T = T;
    a.V = V;
    a.W = W;
    a.e_ld = e_ld;
    a.g_ld = g_ld;
    a.scale = scale;
    a.stream = V * W * bytes_of(g_format) > kStreamBytes;
    a.R = p.R;
    a.log_lanes = p.log_lanes;
    a.slabs = p.slabs;
    a.share = p.share;
    a.piece = p.piece;
    a.pieces = p.pieces;
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    a.start = reinterpret_cast<int*>(ws);
    a.list = reinterpret_cast<int2*>(ws + p.list);
    a.parts = reinterpret_cast<double*>(ws + p.parts);
    FP8T_BY_FORMATS(launch_bwd, e_format, g_format, a, stream)
    return launch_status();
}
