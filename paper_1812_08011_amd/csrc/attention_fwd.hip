// Attention forward on the matrix cores.
//
// A workgroup owns a tile of rows -- (query, query head of a group) pairs, the
// heads of a group beside each other, so that one pass over a key head's keys
// and values serves them all -- and streams key tiles through LDS.  One pass:
// S^T = K Q^T per 32 keys, p = 2^(S c2 - reference) with the row's running
// reference and sum, O^T += V^T P^T with the registers that hold P as the
// operand (the products are transposed for that: a lane owns a row).
//
// The operands of both products are IEEE halves.  FP8 codes are exact in them;
// the FP8 matrix instructions, twice as fast, cut products to 13 bits, which
// moved the log-sum-exps by 3e-5.  p is rounded to a half of its own row's
// scale (2^-12 relative at the largest, absolutely 2^-38 of it): what leaves is
// rounded to 10 bits or 3.  Sums, reference and statistics stay FP32.  Where a
// row's scores are so large that FP32 exponents lose their fraction, they are
// taken from one of them first (kFar).
#include "attn_fwd.h"
#include "attn_image.h"

namespace fp8t {
namespace {

constexpr int kThreads = 256;
// p is held times 2^13 (relative to the row's largest when its reference was set)
// and may grow to 2^15.9 before the reference moves (the largest half is 2^16
// less 32).  With 2^7, half a percent faster on long prompts, results made of
// keys of small weight lost bits from 2^-21 on; 2^14 costs another half.
constexpr float kBase = 13.0f, kRoom = 15.9f;
// Beyond this an exponent S c2 - reference, one FMA, is off by the rounding of
// the reference, 2^-4 and more of a power of two, for all keys alike: halves
// overflow, or underflow to 0.  A row's scores are then taken from a score.
constexpr float kFar = 0x1p20f;

struct Fmax { __device__ float operator()(float a, float b) const { return fmaxf(a, b); } };
struct Add { __device__ float operator()(float a, float b) const { return a + b; } };

// Key tile in flight: the registers between global memory and LDS.
template <int kBN, int DP, int NT>
struct Stage {
    static constexpr int kK = CodeTile<kBN, DP>::template units<NT>();
    static constexpr int kV = HalfTile<kBN, DP>::template units<NT>();
    uint4 k[kK];
    uint2 v[kV][4];
};

template <int kBN, int DP, bool VEC, int NT>
__device__ __forceinline__ void load_k(Stage<kBN, DP, NT>& s, const uint8_t* k, int64_t ts, int j0, int nk,
                                       int D, int tid) {
#pragma unroll
    for (int u = 0; u < Stage<kBN, DP, NT>::kK; ++u) {
        const int id = tid + u * NT, row = id / (DP / 16), col = id % (DP / 16) * 16;
        s.k[u] = load_codes16<VEC>(k + (int64_t)(j0 + row) * ts, col, D, j0 + row < nk);
    }
}
template <int kBN, int DP, bool VEC, int NT>
__device__ __forceinline__ void load_v(Stage<kBN, DP, NT>& s, const uint8_t* v, int64_t ts, int j0, int nk,
                                       int D, int tid) {
    using HT = HalfTile<kBN, DP>;
#pragma unroll
    for (int u = 0; u < Stage<kBN, DP, NT>::kV; ++u) {
        const int id = tid + u * NT, row = j0 + HT::unit_row(id), col = HT::unit_col(id);
#pragma unroll
        for (int r = 0; r < 4; ++r)
            s.v[u][r] = load_codes8<VEC>(v + (int64_t)(row + r) * ts, col, D, row + r < nk);
    }
}
template <int kBN, int DP, int NT>
__device__ __forceinline__ void store_k(const Stage<kBN, DP, NT>& s, uint8_t* lds, int tid) {
#pragma unroll
    for (int u = 0; u < Stage<kBN, DP, NT>::kK; ++u) {
        const int id = tid + u * NT, row = id / (DP / 16), col = id % (DP / 16) * 16;
        *reinterpret_cast<uint4*>(lds + row * CodeTile<kBN, DP>::kRow + col) = s.k[u];
    }
}
// partial: some row does not see some key of the tile.  Values that are not
// finite are then taken out (a matrix product would let 0 x NaN into rows that
// do not see the key) and their keys noted in `bad`.
template <int kBN, int DP, int NT>
__device__ __forceinline__ void store_v(Stage<kBN, DP, NT>& s, uint8_t* lds, int tid, bool partial,
                                        uint32_t* bad) {
    using HT = HalfTile<kBN, DP>;
#pragma unroll
    for (int u = 0; u < Stage<kBN, DP, NT>::kV; ++u) {
        const int id = tid + u * NT;
        if (partial) {
            const int row = HT::unit_row(id);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const uint32_t nx = nonfinite_bytes(s.v[u][r].x), ny = nonfinite_bytes(s.v[u][r].y);
                if (nx | ny) {
                    atomicOr(bad + (row + r) / 32, 1u << ((row + r) % 32));
                    s.v[u][r].x &= ~nx;
                    s.v[u][r].y &= ~ny;
                }
            }
        }
        HT::store(lds, id, s.v[u]);
    }
}

// What a wave holds of its 32 rows: queries, running sums, statistics.  Lane
// half h of column l % 32 holds rows 8 g + 4 h + r of every result.
template <int DP, int N>
struct FwdRows {
    static constexpr int NC = DP / 32, ND = DP / 32, NK = N / 32;
    using HT = HalfTile<N, DP>;
    Widen widen;
    v8h qf[NC][2];
    v16f o[ND];
    float ref, mu, l, c2;              // reference; the same, 0 before the first key; sum; scale
    float base;                        // the score that the others are taken from
    bool far;                          // some row's is not 0
    uint32_t noted_any;                // keys with values that are not finite came by

    template <bool VEC>
    __device__ __forceinline__ void init(const AttnArgs& a, const uint8_t* q, int h, bool live) {
        c2 = __uint_as_float(in_vgpr(__float_as_uint(a.c2)));
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const uint4 w = load_codes16<VEC>(q, 32 * c + 16 * h, a.D, live);
            qf[c][0] = widen(w.x, w.y);
            qf[c][1] = widen(w.z, w.w);
        }
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[d][r] = 0.0f;
        ref = -INFINITY;
        mu = l = base = 0.0f;
        far = false;
        noted_any = 0;
    }

    // One key tile whose first key is j0 (negative: keys of another sequence
    // first): kf(kt, c) gives the key operand, vl the values in LDS; next() runs
    // once the key operands are used up.  partial: some row does not see some
    // key; a row sees keys [0, lim).  noted: the keys whose values are not
    // finite and left out of vl.
    template <typename KF, typename NEXT>
    __device__ __forceinline__ void step(KF kf, const uint8_t* vl, int j0, int lim, bool partial, int h,
                                         int l31, const uint32_t* noted, NEXT next) {
        const v16f zero = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
        v16f st[NK];
#pragma unroll
        for (int kt = 0; kt < NK; ++kt) {
            st[kt] = zero;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const uint4 w = kf(kt, c);
                st[kt] = mfma_half(widen(w.x, w.y), qf[c][0], st[kt]);
                st[kt] = mfma_half(widen(w.z, w.w), qf[c][1], st[kt]);
            }
        }
        next();
        if (partial) {
            int key = j0 + 4 * h;
            asm volatile("" : "+v"(key));                   // a branch: no selects on whole tiles
#pragma unroll
            for (int kt = 0; kt < NK; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if ((uint32_t)(key + 32 * kt + 8 * (r / 4) + r % 4) >= (uint32_t)lim)
                        st[kt][r] = -INFINITY;
        }
        float top = -INFINITY;
#pragma unroll
        for (int kt = 0; kt < NK; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, st[kt][r]);
        top = both_halves(top, Fmax());
        float mx = (top - base) * c2;
        if (__any(mx - ref > kRoom)) {
            // rows whose reference moves to a far score are taken from that
            const bool moves = __builtin_fabsf(mx) > kFar && mx - kBase > ref && mx < INFINITY;
            if (__builtin_expect(__any(moves), 0)) {
                if (moves) {
                    ref = __builtin_fmaf(base - top, c2, ref);
                    base = top;
                    mx = 0.0f;
                }
                far = true;
            }
            const float nref = fmaxf(ref, mx - kBase);
            const float f = nref == ref ? 1.0f : exp2f(ref - nref);
            ref = nref;
            mu = ref == -INFINITY ? 0.0f : ref;
            l *= f;
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[d][r] *= f;
        }
        if (__builtin_expect(far, 0)) {
            float by = base;
            asm volatile("" : "+v"(by));                    // a branch, as above
#pragma unroll
            for (int kt = 0; kt < NK; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r) st[kt][r] -= by;
        }
#pragma unroll
        for (int kt = 0; kt < NK; ++kt) {
            float p[16];
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                p[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(st[kt][r], c2, -mu));
                l += p[r];
            }
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const v8h pf = to_half8(p + 8 * t);
#pragma unroll
                for (int d = 0; d < ND; ++d)
                    o[d] = mfma_half(HT::frag(vl, 32 * d + l31, 2 * kt + t, h), pf, o[d]);
            }
        }
#pragma unroll
        for (int kt = 0; kt < NK; ++kt) noted_any |= noted[kt];
    }

    // The values that are not finite of the keys noted in `bits`, from key j0
    // on, for the rows that see them.  After the last step: inside it this
    // costs the loop 50 registers.
    __device__ __forceinline__ void add(uint32_t bits, int j0, int lim, int h, const uint8_t* v,
                                        int64_t v_ts, int D) {
        add_noted<ND>(bits, v, v_ts, j0, D, h, [&](int key) { return (uint32_t)key < (uint32_t)lim; },
                      [&](int d, int r, uint32_t c) { o[d][r] += fp8_nonfinite(c); });
    }

    // Whether the sums are finite; those that are not, cleared.
    __device__ __forceinline__ bool finite() const {
        float top = 0.0f;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int r = 0; r < 16; r += 2) top = maximum3_abs(top, o[d][r], o[d][r + 1]);
        return top < INFINITY;
    }
    __device__ __forceinline__ void clear_odd() {
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (!(__builtin_fabsf(o[d][r]) < INFINITY)) o[d][r] = 0.0f;
    }
};

// A workgroup's tile of rows and this lane's row in it.
template <int BM, int RW>              // rows, rows from one wave to the next (0: the same rows)
struct FwdTile {
    Seq sq;
    int64_t tq;
    int row0, row, nrows, hk, hq, slot, lim, lim_lo, lim_hi, wave_hi;
    bool live;
    // false: nothing to do.  Row r sees keys [0, limit(r)); the longest tiles
    // come first.
    __device__ __forceinline__ bool init(const AttnArgs& a, int wave, int l31) {
        hk = blockIdx.x % a.Hkv;
        int tile;
        slot = ordered_slot(a.row_order, blockIdx.x / a.Hkv);
        if (slot < 0) return false;
        sq = load_seq(a, slot_owner(a.cu_q, a.S, a.Tq, a.G, BM, slot, tile));
        nrows = sq.nq * a.G;
        const int ntiles = (nrows + BM - 1) / BM;
        if (tile >= ntiles) return false;
        row0 = (ntiles - 1 - tile) * BM;
        row = row0 + RW * wave + l31;
        live = row < nrows;
        const int i = live ? div_g(a, row) : 0, off = sq.nk - sq.nq;
        auto limit = [&](int i) {
            const int n = a.causal ? i + 1 + off : sq.nk;
            return n < 0 ? 0 : n;
        };
        lim = live ? limit(i) : 0;
        lim_lo = limit(div_g(a, row0));
        lim_hi = limit(div_g(a, row0 + BM < nrows ? row0 + BM - 1 : nrows - 1));
        const int w0 = row0 + RW * wave;
        wave_hi = w0 < nrows ? limit(div_g(a, w0 + 31 < nrows ? w0 + 31 : nrows - 1)) : 0;
        tq = sq.q0 + i;
        hq = hk * a.G + (live ? row - i * a.G : 0);
        return true;
    }
};

// log2 of the sum over its largest term or so: near 0, where floats are finest.
__device__ __forceinline__ float row_lse(const AttnArgs& a, float base, float ref, float l) {
    return __builtin_fmaf(base, a.sm_scale, kAttnLn2 * ((ref + kBase) + log2f(__builtin_ldexpf(l, -(int)kBase))));
}

// A row whose scores are all -Inf is 0 / 0 throughout, its infinite values too.
__device__ __forceinline__ float row_inverse(float l) { return l == 0.0f ? NAN : 1.0f / l; }

// xs: kRowsOut bytes of LDS of the wave's own.
template <int DP, int N, int BM, bool SPLIT>
__device__ __forceinline__ void finish_rows(const AttnArgs& a, const AttnSplit& sp,
                                            const FwdTile<BM, BM == 128 ? 32 : 0>& t,
                                            const FwdRows<DP, N>& x, float base, float ref, float l, int lane,
                                            void* xs) {
    const int h = lane >> 5;
    if constexpr (SPLIT) {
        const int64_t part = (int64_t)blockIdx.y * gridDim.x + (int64_t)t.slot * a.Hkv + t.hk;
        const int64_t pr = part * BM + (t.row - t.row0);
        if (h == 0 && t.live) sp.ml[pr] = make_float4(base, ref, l, 0.0f);
        if constexpr (BM == 32) {                           // few of the rows are there
            if (!t.live) return;
            float* po = sp.o + pr * DP + 4 * h;
#pragma unroll
            for (int d = 0; d < DP / 32; ++d)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *reinterpret_cast<float4*>(po + 32 * d + 8 * q) = make_float4(
                        x.o[d][4 * q], x.o[d][4 * q + 1], x.o[d][4 * q + 2], x.o[d][4 * q + 3]);
        } else {
            rows_out<DP>(static_cast<float*>(xs), x.o, 1.0f, lane, [&](int r, int col, const float* v) {
                const int64_t to = of_lane(pr, r);
                if (__shfl((int)t.live, r)) store_some<FP8T_FMT_F32>(sp.o + to * DP + col, 8, v);
            });
        }
    } else {
        if (a.lse && h == 0 && t.live)
            a.lse[(int64_t)t.hq * a.Tq + t.tq] = t.lim > 0 ? row_lse(a, base, ref, l) : -INFINITY;
        if (!a.o && !a.o8) return;
        // a row that sees nothing has sums of +0
        const float inv = t.lim > 0 ? row_inverse(l) : 1.0f;
        const int64_t o = t.tq * a.o_ts + (int64_t)t.hq * a.o_hs;
        const int64_t o8 = t.tq * a.o8_ts + (int64_t)t.hq * a.o8_hs;
        rows_out<DP>(static_cast<float*>(xs), x.o, inv, lane, [&](int r, int col, const float* v) {
            const int64_t at = of_lane(o, r), at8 = of_lane(o8, r);
            const int n = __shfl((int)t.live, r) ? up_to_8(a.D - col) : 0;
            if (n == 0) return;
            if (a.o) store_some<FP8T_FMT_FP16>(a.o + at + col, n, v);
            if (a.o8) {
                float y[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = v[i] * a.o8_scale;
                store_some<FP8T_FMT_FP8>(a.o8 + at8 + col, n, y);
            }
        });
    }
}

// 128 rows, 32 per wave; key tiles come from their image by direct loads into
// LDS, one tile ahead.
//
// Bound by the matrix cores: 550 GFLOP (16384 causal tokens, 8 heads of 128, 2
// key heads) in 551 us, 998 TFLOP/s, where a large half-precision product
// reaches 1138; without the softmax's instructions between them the same matrix
// instructions took 470 us.  275 GFLOP over 8192 tokens: 282 us.  D 64: 46
// GFLOP of mixed lengths in 77 us, the vector ALUs busy for 60% of it and the
// matrix cores for 28% (D 128: 55% and 48%).  With D above 64 a row tile of 128
// keeps 2 waves per SIMD (190 registers a lane), a third spills; with D up to 64
// it is 3 (166).  A third buffer in LDS changed nothing.
template <int DP, bool VEC, bool SPLIT>
__global__ __launch_bounds__(kThreads, 2) void attn_fwd_image_kernel(AttnArgs a, AttnSplit sp) {
    using I = FwdImage<DP>;
    constexpr int N = I::N;
    __shared__ __attribute__((aligned(16))) uint8_t lds[2 * I::kBytes];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int l31 = lane & 31, h = lane >> 5;
    FwdTile<128, 32> t;
    if (!t.init(a, wave, l31)) return;
    // tiles of the packed keys that hold some of [k0, k0 + lim_hi)
    const int first = (int)(t.sq.k0 / N), j00 = (int)((int64_t)first * N - t.sq.k0);
    int t0 = 0, t1 = t.lim_hi > 0 ? (t.lim_hi - j00 + N - 1) / N : 0;
    if (SPLIT) {
        t0 = blockIdx.y * sp.per;
        if (blockIdx.y + 1 < gridDim.y && t0 + sp.per < t1) t1 = t0 + sp.per;
    }
    const uint8_t* image = a.key_image + ((int64_t)t.hk * a.key_tiles + first) * I::kBytes;
    const uint8_t* vp = a.v.p + t.sq.k0 * a.v.ts + (int64_t)t.hk * a.v.hs;
    if (t0 < t1) image_to_lds<I::kBytes, 4>(image + (int64_t)t0 * I::kBytes, lds, wave, lane);
    FwdRows<DP, N> x;
    x.template init<VEC>(a, a.q.p + t.tq * a.q.ts + (int64_t)t.hq * a.q.hs, h, t.live);
    for (int n = t0; n < t1; ++n) {
        const uint8_t* buf = lds + ((n - t0) & 1) * I::kBytes;
        image_barrier();
        if (n + 1 < t1)
            image_to_lds<I::kBytes, 4>(image + (int64_t)(n + 1) * I::kBytes,
                                       lds + ((n + 1 - t0) & 1) * I::kBytes, wave, lane);
        const int j0 = j00 + n * N;
        if (j0 >= t.wave_hi) continue;
        x.step([&](int kt, int c) { return I::CT::frag(buf, 32 * kt + l31, c, h); }, buf + I::kV, j0, t.lim,
               j0 < 0 || j0 + N > t.lim_lo, h, l31, reinterpret_cast<const uint32_t*>(buf + I::kNoted),
               []() {});
    }
    if (__builtin_expect(__any(x.noted_any != 0), 0)) {
#pragma unroll 1
        for (int i = t0 * (N / 32); i < t1 * (N / 32); ++i) {
            const uint8_t* at = image + (int64_t)(i / (N / 32)) * I::kBytes + I::kNoted;
            x.add(reinterpret_cast<const uint32_t*>(at)[i % (N / 32)], j00 + 32 * i, t.lim, h, vp, a.v.ts, a.D);
        }
    }
    const float l = both_halves(x.l, Add());
    __syncthreads();                                        // the buffers are free
    finish_rows<DP, N, 128, SPLIT>(a, sp, t, x, x.base, x.ref, l, lane, lds + wave * kRowsOut);
}

// KW = 1: 128 rows, 32 per wave, every wave walks all key tiles (shared in
// LDS, double-buffered).  KW = 4: 32 rows, each wave walks every fourth key
// tile by itself and the waves' results are joined in LDS -- for calls with
// few rows, where the keys are what there is to share out.
// SPLIT: the key tiles are shared out over gridDim.y workgroups, whose partial
// results go to the workspace.
//
// Few rows are bound by the keys and values read (44 MB for 8 tokens, 32 heads
// and 8 key heads of 128, over 21 thousand keys: 23 us, 1.9 TB/s, and 6 us for
// the join; a copy of that size would take 9 us) and by the latency of a
// workgroup's start, first loads and join: 11 us where there is one key.  Many
// short sequences (24 of up to 96 tokens, 16 heads of 64) take 10 us, nearly
// all of it that latency.  KW = 4 with D above 64 takes all 256 registers and 64
// to 92 bytes of scratch a lane: the next tile's keys and values are in flight
// beside the queries and 64 sums.
template <int DP, int KW, bool VEC, bool SPLIT>
__global__ __launch_bounds__(kThreads, 2) void attn_fwd_kernel(AttnArgs a, AttnSplit sp) {
    constexpr int NT = kThreads / KW, BM = 128 / KW, kBN = KW == 1 ? attn_keys(DP) : attn_keys(DP) / 2;
    constexpr int NB = KW == 1 ? 2 : 4;                     // LDS buffers: double, or one per wave
    constexpr int NC = DP / 32, ND = DP / 32, NK = kBN / 32;
    using CT = CodeTile<kBN, DP>;
    using HT = HalfTile<kBN, DP>;
    constexpr int kKeys = KW == 1 ? NB * CT::kBytes : 0;    // KW = 4: keys go straight to registers
    constexpr int kTiles = kKeys + NB * HT::kBytes, kJoin = KW == 1 ? 0 : 3 * ND * 16 * 64 * 4;
    __shared__ __attribute__((aligned(16))) uint8_t lds[kTiles > kJoin ? kTiles : kJoin];
    uint8_t* const ks = lds;
    uint8_t* const vs = lds + kKeys;
    __shared__ uint32_t bad[4][NK];
    static_assert(sizeof(lds) >= (KW == 1 ? 4 : 1) * kRowsOut && 2 * FwdImage<DP>::kBytes >= 4 * kRowsOut,
                  "the results' way out fits the buffers");
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, l31 = lane & 31, h = lane >> 5;
    FwdTile<BM, KW == 1 ? 32 : 0> w;
    if (!w.init(a, wave, l31)) return;
    const Seq& sq = w.sq;
    int t0 = 0, t1 = (w.lim_hi + kBN - 1) / kBN;
    if (SPLIT) {
        t0 = blockIdx.y * sp.per;
        if (blockIdx.y + 1 < gridDim.y && t0 + sp.per < t1) t1 = t0 + sp.per;
    }
    const uint8_t* kp = a.k.p + sq.k0 * a.k.ts + (int64_t)w.hk * a.k.hs;
    const uint8_t* vp = a.v.p + sq.k0 * a.v.ts + (int64_t)w.hk * a.v.hs;
    FwdRows<DP, kBN> x;
    x.template init<VEC>(a, a.q.p + w.tq * a.q.ts + (int64_t)w.hq * a.q.hs, h, w.live);
    auto is_partial = [&](int t) { return (t + 1) * kBN > w.lim_lo; };

    Stage<kBN, DP, NT> sg;
    if constexpr (KW == 1) {
        if (tid < 4 * NK) bad[tid / NK][tid % NK] = 0u;
        __syncthreads();
        if (t0 < t1) {
            load_k<kBN, DP, VEC>(sg, kp, a.k.ts, t0 * kBN, sq.nk, a.D, tid);
            load_v<kBN, DP, VEC>(sg, vp, a.v.ts, t0 * kBN, sq.nk, a.D, tid);
            store_k(sg, ks, tid);
            store_v(sg, vs, tid, is_partial(t0), bad[0]);
        }
        __syncthreads();
        for (int t = t0; t < t1; ++t) {
            const int b = (t - t0) & 1, q = (t - t0) % 3;
            if (t + 1 < t1) {
                load_k<kBN, DP, VEC>(sg, kp, a.k.ts, (t + 1) * kBN, sq.nk, a.D, tid);
                load_v<kBN, DP, VEC>(sg, vp, a.v.ts, (t + 1) * kBN, sq.nk, a.D, tid);
            }
            if (t * kBN < w.wave_hi) {
                const uint8_t* kl = ks + b * CT::kBytes;
                x.step([&](int kt, int c) { return CT::frag(kl, 32 * kt + l31, c, h); },
                       vs + b * HT::kBytes, t * kBN, w.lim, is_partial(t), h, l31, bad[q], []() {});
            }
            // noted keys: slot q is read here, the next one written, the one
            // read in the last step cleared
            if (tid < NK) bad[(q + 2) % 3][tid] = 0u;
            if (t + 1 < t1) {
                store_k(sg, ks + (b ^ 1) * CT::kBytes, tid);
                store_v(sg, vs + (b ^ 1) * HT::kBytes, tid, is_partial(t + 1), bad[(q + 1) % 3]);
            }
            __syncthreads();
        }
    } else {
        uint8_t* vl = vs + wave * HT::kBytes;
        uint4 kf[NK][NC];
        auto load = [&](int t) {
#pragma unroll
            for (int kt = 0; kt < NK; ++kt) {
                const int j = t * kBN + 32 * kt + l31;
#pragma unroll
                for (int c = 0; c < NC; ++c)
                    kf[kt][c] = load_codes16<VEC>(kp + (int64_t)j * a.k.ts, 32 * c + 16 * h, a.D,
                                                  j < sq.nk);
            }
            load_v<kBN, DP, VEC>(sg, vp, a.v.ts, t * kBN, sq.nk, a.D, lane);
        };
        // a wave works by itself here: its LDS accesses are ordered
        auto fence = [&]() {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        };
        if (t0 + wave < t1) load(t0 + wave);
        for (int t = t0 + wave; t < t1; t += KW) {
            fence();
            if (lane < NK) bad[wave][lane] = 0u;
            fence();
            store_v(sg, vl, lane, is_partial(t), bad[wave]);
            fence();
            x.step([&](int kt, int c) { return kf[kt][c]; }, vl, t * kBN, w.lim, is_partial(t), h, l31,
                   bad[wave], [&]() {
                       if (t + KW < t1) load(t + KW);
                   });
        }
    }
    float l = both_halves(x.l, Add()), base = x.base, ref = x.ref;
    // A value that is not finite in a tile that every row sees has made its
    // column's sums Inf, or NaN where its p underflowed (0 x Inf): they start
    // again from 0.
    const bool odd = !x.finite() && l == l;
    if (__builtin_expect(__any(x.noted_any != 0 || odd), 0)) {
        if (odd) x.clear_odd();
        // the wave's tiles again, 32 keys at a time looked at by the whole wave
#pragma unroll 1
        for (int t = t0 + (KW > 1 ? wave : 0); t < t1; t += KW)
#pragma unroll 1
            for (int j0 = t * kBN; j0 < (t + 1) * kBN && j0 < sq.nk; j0 += 32) {
                uint32_t some = 0;
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    const uint4 u = load_codes16<VEC>(vp + (int64_t)(j0 + l31) * a.v.ts, 32 * c + 16 * h, a.D,
                                                      j0 + l31 < sq.nk);
                    some |= nonfinite_in(u.x) | nonfinite_in(u.y) | nonfinite_in(u.z) | nonfinite_in(u.w);
                }
                const uint64_t rows = __ballot((some & 0x80808080u) != 0);
                x.add((uint32_t)rows | (uint32_t)(rows >> 32), j0, w.lim, h, vp, a.v.ts, a.D);
            }
    }

    if constexpr (KW > 1) {
        // join the waves: references first, then the scaled sums
        __shared__ float bases[KW][32], refs[KW][32], ls[KW][32];
        __syncthreads();
        if (h == 0) {
            bases[wave][l31] = base;
            refs[wave][l31] = ref;
            ls[wave][l31] = l;
        }
        __syncthreads();
        float bm = bases[0][l31], m = refs[0][l31];
#pragma unroll
        for (int v = 1; v < KW; ++v) {
            const float bv = bases[v][l31], rv = refs[v][l31];
            if (part_above(bv, rv, bm, m, a.c2) > 0.0f) {
                bm = bv;
                m = rv;
            }
        }
        l = 0.0f;
#pragma unroll
        for (int v = 0; v < KW; ++v)
            l += ls[v][l31] * part_weight(bases[v][l31], refs[v][l31], bm, m, a.c2);
        const float f = part_weight(base, ref, bm, m, a.c2);
        float* xs = reinterpret_cast<float*>(vs);           // [wave - 1][register][lane]
        if (wave) {
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    xs[(((wave - 1) * ND + d) * 16 + r) * 64 + lane] = x.o[d][r] * f;
        }
        __syncthreads();
        if (wave) return;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                float y = x.o[d][r] * f;
                for (int v = 0; v < KW - 1; ++v) y += xs[((v * ND + d) * 16 + r) * 64 + lane];
                x.o[d][r] = y;
            }
        base = bm;
        ref = m;
    }
    // KW = 1: the last step ended at a barrier; KW = 4: one wave is left
    finish_rows<DP, kBN, BM, SPLIT>(a, sp, w, x, base, ref, l, lane, lds + (KW == 1 ? wave * kRowsOut : 0));
}

// Joins the partial results of a tile's key ranges, in their order: a wave per
// row, a lane for every 64th entry.  Latency-bound: 6 to 8 us where the rows are
// few.
template <int DP, int BM>
__global__ __launch_bounds__(kThreads) void attn_join_kernel(AttnArgs a, AttnSplit sp) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int hk = blockIdx.x % a.Hkv;
    int tile;
    const Seq sq = load_seq(a, slot_owner(a.cu_q, a.S, a.Tq, a.G, BM, blockIdx.x / a.Hkv, tile));
    const int nrows = sq.nq * a.G, ntiles = (nrows + BM - 1) / BM;
    if (tile >= ntiles) return;
    tile = ntiles - 1 - tile;
    const int rr = blockIdx.y * (kThreads / 64) + wave, row = tile * BM + rr;
    if (rr >= BM || row >= nrows) return;
    const int i = div_g(a, row), off = sq.nk - sq.nq, lim = a.causal ? i + 1 + off : sq.nk;
    // lane z takes range z's reference and sum (there are at most 64).  A range
    // without a key has neither; one whose scores are all NaN has a sum of NaN,
    // which has to come through.
    const int64_t stride = (int64_t)gridDim.x * BM, first = (int64_t)blockIdx.x * BM + rr;
    const float4 ml = lane < sp.n ? sp.ml[lane * stride + first] : make_float4(0.0f, -INFINITY, 0.0f, 0.0f);
    const bool some = ml.y != -INFINITY || ml.z != 0.0f;
    float bm = ml.x, m = ml.y;
#pragma unroll
    for (int d = 32; d; d >>= 1) {
        const float bv = __shfl_xor(bm, d), rv = __shfl_xor(m, d);
        if (part_above(bv, rv, bm, m, a.c2) > 0.0f) {
            bm = bv;
            m = rv;
        }
    }
    bm = __shfl(bm, 0);                                     // of equal ones the same for all
    m = __shfl(m, 0);
    const float f = part_weight(ml.x, ml.y, bm, m, a.c2);
    float l = some ? ml.z * f : 0.0f;
#pragma unroll
    for (int d = 32; d; d >>= 1) l += __shfl_xor(l, d);
    float o[2] = {0.0f, 0.0f};
#pragma unroll 4
    for (int z = 0; z < sp.n; ++z) {
        if (!__shfl((int)some, z)) continue;
        const float w = __shfl(f, z);
#pragma unroll
        for (int u = 0; u < DP / 64; ++u) o[u] += sp.o[(z * stride + first) * DP + 64 * u + lane] * w;
    }
    const int64_t t = sq.q0 + i;
    const int hq = hk * a.G + row - i * a.G;
    const float inv = row_inverse(l);
#pragma unroll
    for (int u = 0; u < DP / 64; ++u) {
        const int d = 64 * u + lane;
        const float x = lim > 0 ? o[u] * inv : 0.0f;
        if (d >= a.D) continue;
        if (a.o) a.o[t * a.o_ts + hq * a.o_hs + d] = f32_to_fp16_rn(x);
        if (a.o8) a.o8[t * a.o8_ts + hq * a.o8_hs + d] = (uint8_t)f32_to_fp8(x * a.o8_scale);
    }
    if (a.lse && lane == 0)
        a.lse[(int64_t)hq * a.Tq + t] = lim > 0 ? row_lse(a, bm, m, l) : -INFINITY;
}

template <int DP, bool VEC>
void launch(const AttnArgs& a, const AttnFwdPlan& p, const AttnSplit& sp, hipStream_t stream) {
    const dim3 grid((unsigned)(a.Hkv * p.slots), (unsigned)p.splits), block(kThreads);
    const bool split = p.splits > 1;
    if (p.image) {
        attn_fwd_image_launch(a, VEC, DP, stream);
        if (split) hipLaunchKernelGGL((attn_fwd_image_kernel<DP, VEC, true>), grid, block, 0, stream, a, sp);
        else hipLaunchKernelGGL((attn_fwd_image_kernel<DP, VEC, false>), grid, block, 0, stream, a, sp);
    } else if (p.BM == 32) {
        if (split) hipLaunchKernelGGL((attn_fwd_kernel<DP, 4, VEC, true>), grid, block, 0, stream, a, sp);
        else hipLaunchKernelGGL((attn_fwd_kernel<DP, 4, VEC, false>), grid, block, 0, stream, a, sp);
    } else {
        if (split) hipLaunchKernelGGL((attn_fwd_kernel<DP, 1, VEC, true>), grid, block, 0, stream, a, sp);
        else hipLaunchKernelGGL((attn_fwd_kernel<DP, 1, VEC, false>), grid, block, 0, stream, a, sp);
    }
    if (split && p.BM == 32)
        hipLaunchKernelGGL((attn_join_kernel<DP, 32>), dim3(grid.x, 8), block, 0, stream, a, sp);
    else if (split)
        hipLaunchKernelGGL((attn_join_kernel<DP, 128>), dim3(grid.x, 32), block, 0, stream, a, sp);
}

}  // namespace

// Which kernel, by the packed rows (query, head of the group) of the longest
// sequence.  Measured with 16 query and 4 key/value heads unless stated:
//
// * up to 32 rows: the kernel whose waves share out the keys of 32 rows.  8
//   sequences with 2048 keys, 4 rows: 12 us against 31 us (D 64) and 16
//   against 30 us (D 128) for the kernel of 128 rows; with 64 and 128 rows the
//   two lie within a third of each other, either way by the number of keys.
// * 4096 rows and more: keys from tiles laid out beforehand, which 32 row tiles
//   or more read then.  4 sequences of 4096 tokens, D 128: 282 us, directly
//   from the operands 318 us; 16 heads without groups: 296 and 313 us; 1024
//   tokens over 8192 keys: 292 and 320 us.  With 2048 rows the layout costs what
//   it saves (64.5 and 63.9 us) and below that more (1024 rows: 23 and 18 us).
// * D up to 64 pays for 64 columns, above for 128: half the products and half
//   the loads.
//
// The keys are shared out over workgroups where the rows leave CUs idle, until
// there are 4 workgroups per CU (2 for the kernel of few rows: 27 us for 8
// tokens over long histories where 4 take 31 us, a longer join), with at least
// 8 steps of keys each: with 16, 64 rows over 4 x 4096 keys take 36 us in place
// of 23 us; with 4, 4 rows over 8 x 2048 keys take 15 us in place of 12 us.
AttnFwdPlan attn_fwd_plan(int64_t S, int64_t Tq, int64_t Tk, int64_t max_q, int64_t max_k, int64_t Hq,
                          int64_t Hkv, int64_t D) {
    AttnFwdPlan p = {};
    const int64_t G = Hkv ? Hq / Hkv : 1;
    max_q = hint(max_q, G);
    max_k = hint(max_k, 1);
    p.DP = D <= 64 ? 64 : 128;
    p.BM = max_q * G <= 32 ? 32 : 128;
    p.slots = slots(S, Tq, G, p.BM);
    p.image = p.BM == 128 && max_q * G >= 4096 && Tk > 0;     // no keys: no tiles to launch for
    const int64_t image = p.image ? image_tiles(Tk, attn_keys(p.DP)) * Hkv *
                                        (p.DP == 64 ? FwdImage<64>::kBytes : FwdImage<128>::kBytes)
                                  : 0;
    const int64_t tiles_q = (max_q * G + p.BM - 1) / p.BM;
    int64_t groups = p.slots < S * tiles_q ? p.slots : S * tiles_q;
    groups *= Hkv;
    const int kBN = p.BM == 32 ? attn_keys(p.DP) / 2 : attn_keys(p.DP);
    const int64_t tiles_k = (max_k + kBN - 1) / kBN;
    const int64_t want = (p.BM == 32 ? 2 : 4) * (int64_t)device_cus(), least = 8;
    int64_t n = groups > 0 && groups * 2 <= want ? want / groups : 1;
    if (n > tiles_k / least) n = tiles_k / least;
    if (n > 64) n = 64;
    p.splits = n > 1 ? (int)n : 1;
    p.per = (int)((tiles_k + p.splits - 1) / p.splits);
    p.order = p.image && S > 1;
    p.fits = p.slots * Hkv <= kAttnGrid &&
             (!p.image || image_tiles(Tk, attn_keys(p.DP)) * Hkv < kAttnGrid);
    p.image_bytes = (size_t)image + (p.order ? (p.slots * 4 + 15) / 16 * 16 : 0);
    p.bytes = p.image_bytes +
              (p.splits > 1 ? (size_t)p.splits * p.slots * Hkv * p.BM * (p.DP * 4 + sizeof(float4)) : 0);
    return p;
}

void attn_fwd_launch(AttnArgs a, const AttnFwdPlan& p, bool vec, void* workspace, hipStream_t stream) {
    AttnSplit sp = {};
    a.key_image = static_cast<uint8_t*>(workspace);
    a.key_tiles = image_tiles(a.Tk, attn_keys(p.DP));
    if (p.image && p.order)
        a.row_order = reinterpret_cast<int*>(a.key_image + p.image_bytes - (p.slots * 4 + 15) / 16 * 16);
    if (p.splits > 1) {
        const int64_t rows = (int64_t)p.splits * p.slots * a.Hkv * p.BM;
        sp.o = reinterpret_cast<float*>(a.key_image + p.image_bytes);
        sp.ml = reinterpret_cast<float4*>(sp.o + rows * p.DP);
        sp.n = p.splits;
        sp.per = p.per;
    }
    if (p.DP == 64) {
        if (vec) launch<64, true>(a, p, sp, stream);
        else launch<64, false>(a, p, sp, stream);
    } else {
        if (vec) launch<128, true>(a, p, sp, stream);
        else launch<128, false>(a, p, sp, stream);
    }
}

}  // namespace fp8t
