// Builds the images (attn_image.h).  A workgroup builds one tile of one head in
// LDS and writes it out 16 bytes a thread.
//
// Bound by what they read and write.  8192 tokens of 128: keys of 4 heads for
// the forward pass 7 us (8 MB in, 13 out), keys for the backward pass 11 us (8
// in, 18 out), queries and errors of 16 heads 35 us (67 MB with o in, 105 out:
// 4.9 TB/s).
#include "attn_image.h"

namespace fp8t {
namespace {

constexpr int kThreads = 256;

// Four rows x eight columns of the tile that starts at token t0.
template <int N, int DP, bool VEC>
__device__ __forceinline__ void load_unit(uint2* w, const AttnRows& r, int64_t head, int64_t t0, int64_t T,
                                          int D, int u) {
    const int row = HalfTile<N, DP>::unit_row(u), col = HalfTile<N, DP>::unit_col(u);
    const uint8_t* p = r.p + head * r.hs;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        w[i] = load_codes8<VEC>(p + (t0 + row + i) * r.ts, col, D, t0 + row + i < T);
}
template <int N, int DP>
__device__ __forceinline__ void store_codes(const uint2* w, uint8_t* lds, int u) {
    const int row = HalfTile<N, DP>::unit_row(u), col = HalfTile<N, DP>::unit_col(u);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        *reinterpret_cast<uint2*>(lds + (row + i) * CodeTile<N, DP>::kRow + col) = w[i];
}
// Transposed, without the values that are not finite, whose rows are noted.
template <int N, int DP>
__device__ __forceinline__ void store_halves(uint2* w, uint8_t* lds, int u, uint32_t* noted) {
    const int row = HalfTile<N, DP>::unit_row(u);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t nx = nonfinite_bytes(w[i].x), ny = nonfinite_bytes(w[i].y);
        if (nx | ny) {
            atomicOr(noted + (row + i) / 32, 1u << ((row + i) % 32));
            w[i].x &= ~nx;
            w[i].y &= ~ny;
        }
    }
    HalfTile<N, DP>::store(lds, u, w);
}
template <int BYTES>
__device__ __forceinline__ void write_image(const uint8_t* lds, uint8_t* dst) {
    __syncthreads();
    for (int i = threadIdx.x; i < BYTES / 16; i += kThreads)
        reinterpret_cast<uint4*>(dst)[i] = reinterpret_cast<const uint4*>(lds)[i];
}
// Orders the tiles of all sequences by their work, the longest first (a
// counting sort over 256 classes), so that no long tile starts last: with
// sequences of many lengths in one batch the order of the slots leaves the
// card waiting for the last long sequence.  8 sequences of 1 to 8192 tokens, 16
// heads of 64: forward 224 us, in the order of the slots 240; backward 726 and
// 781.  8 causal sequences of 2048, 16 heads of 128: 153 and 164; 606 and 703.
// Sequences of one length gain too, by their causal tiles.  It costs 4 us of
// one workgroup beside the others.  Rows (KEYS false) or keys.  The
// order inside a class is open; no result depends on it.  lds: ORDER ints of
// the workgroup's, where the first slots' work is kept (it takes a search
// through the offsets); the others' is looked up again.
template <bool KEYS, int ORDER>
__device__ __forceinline__ void order_tiles(const AttnArgs& a, int* order, uint8_t* lds) {
    constexpr int kTile = KEYS ? kAttnDkvKeys : kAttnRows;
    static_assert(kThreads == 256, "a thread per class");
    __shared__ int count[257], sums[kThreads / 64];
    __shared__ int top;
    int* kept = reinterpret_cast<int*>(lds);
    const int tid = threadIdx.x;
    const int64_t* cu = KEYS ? a.cu_k : a.cu_q;
    const int64_t T = KEYS ? a.Tk : a.Tq, mult = KEYS ? 1 : a.G;
    const int n = (int)(T * mult / kTile + a.S);
    // keys that the tile's last row sees, or queries that see the tile's first
    // key; -1: an empty slot
    auto look_up = [&](int slot) {
        int tile;
        const Seq sq = load_seq(a, slot_owner(cu, a.S, T, mult, kTile, slot, tile));
        const int64_t len = KEYS ? sq.nk : (int64_t)sq.nq * a.G, first = (int64_t)tile * kTile;
        if (first >= len) return -1;
        const int off = sq.nk - sq.nq;
        if (KEYS) {
            const int64_t lo = a.causal && first - off > 0 ? first - off : 0;
            return lo < sq.nq ? (int)(sq.nq - lo) : 0;
        }
        // row tiles run backwards in their slots
        const int64_t ntiles = (len + kTile - 1) / kTile, t = ntiles - 1 - tile;
        const int64_t last = (t + 1) * kTile < len ? (t + 1) * kTile - 1 : len - 1;
        const int64_t lim = a.causal ? div_g(a, (int)last) + 1 + off : sq.nk;
        return lim > 0 ? (int)lim : 0;
    };
    count[tid] = 0;
    if (tid == 0) {
        count[256] = 0;
        top = 1;
    }
    __syncthreads();
    int most = 1;
    for (int i = tid; i < n; i += kThreads) {
        const int w = look_up(i);
        if (i < ORDER) kept[i] = w;                         // read by this thread only
        most = max(most, w);
    }
    atomicMax(&top, most);
    __syncthreads();
    const float per = 255.0f / (float)top;
    auto work = [&](int i) { return i < ORDER ? kept[i] : look_up(i); };
    auto place = [&](int w) { return w < 0 ? 256 : 255 - (int)((float)w * per); };
    for (int i = tid; i < n; i += kThreads) atomicAdd(&count[place(work(i))], 1);
    __syncthreads();
    // each class starts where the ones before it end
    const int own = count[tid];
    int sum = own;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int below = __shfl_up(sum, d);
        if ((tid & 63) >= d) sum += below;
    }
    if ((tid & 63) == 63) sums[tid >> 6] = sum;
    __syncthreads();
    for (int i = 0; i < tid >> 6; ++i) sum += sums[i];
    count[tid] = sum - own;
    if (tid == 255) count[256] = sum;
    __syncthreads();
    for (int i = tid; i < n; i += kThreads) {
        const int w = work(i);
        order[atomicAdd(&count[place(w)], 1)] = w < 0 ? -1 : i;
    }
}

template <int DP, bool VEC>
__global__ __launch_bounds__(kThreads) void fwd_image_kernel(AttnArgs a) {
    using I = FwdImage<DP>;
    __shared__ __attribute__((aligned(16))) uint8_t lds[I::kBytes];
    if (a.row_order && blockIdx.x == 0) {
        order_tiles<false, I::kBytes / 4>(a, a.row_order, lds);
        return;
    }
    const int block = blockIdx.x - (a.row_order ? 1 : 0);
    const int tid = threadIdx.x, hk = block % a.Hkv, t = block / a.Hkv;
    const int64_t t0 = (int64_t)t * I::N;
    uint32_t* noted = reinterpret_cast<uint32_t*>(lds + I::kNoted);
    if (tid < 4) noted[tid] = 0u;
#pragma unroll
    for (int u = 0; u < I::N * (DP / 16) / kThreads; ++u) {
        const int id = tid + u * kThreads, row = id / (DP / 16), col = id % (DP / 16) * 16;
        *reinterpret_cast<uint4*>(lds + row * I::CT::kRow + col) = load_codes16<VEC>(
            a.k.p + (t0 + row) * a.k.ts + (int64_t)hk * a.k.hs, col, a.D, t0 + row < a.Tk);
    }
    uint2 w[4];
    load_unit<I::N, DP, VEC>(w, a.v, hk, t0, a.Tk, a.D, tid);
    __syncthreads();
    store_halves<I::N, DP>(w, lds + I::kV, tid, noted);
    write_image<I::kBytes>(lds, a.key_image + ((int64_t)hk * a.key_tiles + t) * I::kBytes);
}

template <int DP, bool VEC>
__global__ __launch_bounds__(kThreads) void key_image_kernel(AttnArgs a) {
    using I = KeyImage<DP>;
    constexpr int U = (I::N / 4) * (DP / 8), VU = I::N * (DP / 16) / kThreads;
    __shared__ __attribute__((aligned(16))) uint8_t lds[I::kBytes];
    const int tid = threadIdx.x;
    if (a.row_order && blockIdx.x < 2) {
        if (blockIdx.x == 0) order_tiles<false, I::kBytes / 4>(a, a.row_order, lds);
        else order_tiles<true, I::kBytes / 4>(a, a.key_order, lds);
        return;
    }
    const int block = blockIdx.x - (a.row_order ? 2 : 0);
    const int hk = block % a.Hkv, t = block / a.Hkv;
    const int64_t t0 = (int64_t)t * I::N;
    uint32_t* noted = reinterpret_cast<uint32_t*>(lds + I::kNoted);
    if (tid < 4) noted[tid] = 0u;
#pragma unroll
    for (int u = 0; u < VU; ++u) {
        const int id = tid + u * kThreads, row = id / (DP / 16), col = id % (DP / 16) * 16;
        *reinterpret_cast<uint4*>(lds + I::kV + row * I::CT::kRow + col) = load_codes16<VEC>(
            a.v.p + (t0 + row) * a.v.ts + (int64_t)hk * a.v.hs, col, a.D, t0 + row < a.Tk);
    }
    __syncthreads();
    uint2 w[4];
    if (tid < U) {
        load_unit<I::N, DP, VEC>(w, a.k, hk, t0, a.Tk, a.D, tid);
        store_codes<I::N, DP>(w, lds, tid);
        store_halves<I::N, DP>(w, lds + I::kT, tid, noted);
    }
    write_image<I::kBytes>(lds, a.key_image + ((int64_t)hk * a.key_tiles + t) * I::kBytes);
}

// Also delta = <e, o> of every row; o has the 10 bits that it was stored with.
template <int DP, bool VEC>
__global__ __launch_bounds__(kThreads) void query_image_kernel(AttnArgs a, int vec_o) {
    using I = QueryImage<DP>;
    constexpr int U = (I::N / 4) * (DP / 8);
    __shared__ __attribute__((aligned(16))) uint8_t lds[I::kBytes];
    const int tid = threadIdx.x, hq = blockIdx.x % a.Hq, t = blockIdx.x / a.Hq;
    const int64_t t0 = (int64_t)t * I::N;
    uint32_t* noted = reinterpret_cast<uint32_t*>(lds + I::kNoted);
    if (tid < 4) noted[tid] = 0u;
    __syncthreads();
    if (tid < 2 * U) {
        uint2 w[4];
        const int is_e = tid >= U, u = tid % U;
        load_unit<I::N, DP, VEC>(w, is_e ? a.e : a.q, hq, t0, a.Tq, a.D, u);
        store_codes<I::N, DP>(w, lds + is_e * I::kE, u);
        store_halves<I::N, DP>(w, lds + (is_e ? I::kET : I::kQT), u, noted + is_e);
    }
    __syncthreads();
    // 16 lanes per row, 8 entries each
#pragma unroll
    for (int pass = 0; pass < 2; ++pass) {
        const int row = pass * 16 + tid / 16, d0 = tid % 16 * 8;
        const bool live = t0 + row < a.Tq;
        uint2 w = make_uint2(0, 0);
        if (d0 < DP) w = *reinterpret_cast<const uint2*>(lds + I::kE + row * I::CT::kRow + d0);
        const uint16_t* o = a.o + (t0 + row) * a.o_ts + (int64_t)hq * a.o_hs;
        uint32_t oc[4] = {0, 0, 0, 0};
        if (live && d0 < a.D) {
            if (vec_o) {
                const uint4 x = *reinterpret_cast<const uint4*>(o + d0);
                oc[0] = x.x;
                oc[1] = x.y;
                oc[2] = x.z;
                oc[3] = x.w;
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (d0 + i < a.D) oc[i / 2] |= (uint32_t)o[d0 + i] << (16 * (i % 2));
            }
        }
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float e = fp8_to_f32<0>(((i < 4 ? w.x : w.y) >> (8 * (i % 4))) & 0xFFu);
            s = __builtin_fmaf(e, fp16_to_f32((oc[i / 2] >> (16 * (i % 2))) & 0xFFFFu), s);
        }
#pragma unroll
        for (int d = 8; d; d >>= 1) s += __shfl_xor(s, d);
        if (tid % 16 == 0) {
            float l = INFINITY;                             // no such row, or one that sees nothing: p = 0
            if (live) {
                a.delta[(int64_t)hq * a.Tq + t0 + row] = s;
                const float x = a.lse[(int64_t)hq * a.Tq + t0 + row];
                if (x != -INFINITY) l = x * kAttnLog2e - (float)kAttnPUp;
            }
            *reinterpret_cast<float*>(lds + I::lse(row / 4) + 4 * (row % 4)) = l;
            *reinterpret_cast<float*>(lds + I::delta(row / 4) + 4 * (row % 4)) = live ? -s : 0.0f;
        }
    }
    write_image<I::kBytes>(lds, a.query_image + ((int64_t)hq * a.query_tiles + t) * I::kBytes);
}

template <int DP, bool VEC>
void launch_bwd(const AttnArgs& a, bool vec_o, hipStream_t stream) {
    const int64_t nk = a.key_tiles * a.Hkv + (a.row_order ? 2 : 0);
    if (nk) hipLaunchKernelGGL((key_image_kernel<DP, VEC>), dim3((unsigned)nk), dim3(kThreads), 0, stream, a);
    if (a.query_tiles)
        hipLaunchKernelGGL((query_image_kernel<DP, VEC>), dim3((unsigned)(a.query_tiles * a.Hq)),
                           dim3(kThreads), 0, stream, a, (int)vec_o);
}

}  // namespace

void attn_fwd_image_launch(const AttnArgs& a, bool vec, int DP, hipStream_t stream) {
    const dim3 grid((unsigned)(a.key_tiles * a.Hkv + (a.row_order ? 1 : 0))), block(kThreads);
    if (DP == 64) {
        if (vec) hipLaunchKernelGGL((fwd_image_kernel<64, true>), grid, block, 0, stream, a);
        else hipLaunchKernelGGL((fwd_image_kernel<64, false>), grid, block, 0, stream, a);
    } else {
        if (vec) hipLaunchKernelGGL((fwd_image_kernel<128, true>), grid, block, 0, stream, a);
        else hipLaunchKernelGGL((fwd_image_kernel<128, false>), grid, block, 0, stream, a);
    }
}

void attn_bwd_image_launch(const AttnArgs& a, bool vec, int DP, hipStream_t stream) {
    const bool vec_o = a.D % 8 == 0 && aligned(a.o, 16) && a.o_ts % 8 == 0 && a.o_hs % 8 == 0;
    if (DP == 64) {
        if (vec) launch_bwd<64, true>(a, vec_o, stream);
        else launch_bwd<64, false>(a, vec_o, stream);
    } else {
        if (vec) launch_bwd<128, true>(a, vec_o, stream);
        else launch_bwd<128, false>(a, vec_o, stream);
    }
}

}  // namespace fp8t
