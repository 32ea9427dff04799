// bf16 matrix products of the linear layer (y, dx, dW) and of the output layer's cross entropy (scores with their statistics; dx, dW).
#include <algorithm>
#include <atomic>

#include "gemm_bf16_tile.h"
#include "layers_device.h"

namespace rnnt {

namespace {

// What a job covers once the device's row count is known.
struct JobExtent {
    long long M;
    int stages;
};
__device__ __forceinline__ JobExtent job_extent(const GemmJob& g) {
    JobExtent x{g.M, g.stages};
    if (g.limit != GEMM_FIXED) {
        long long n = (long long)*g.count - g.row0;
        n = n < 0 ? 0 : n;
        if (g.limit == GEMM_ROWS_M) x.M = n < x.M ? n : x.M;
        else {
            const long long s = (n + GK - 1) / GK;
            x.stages = s < x.stages ? (int)s : x.stages;
        }
    }
    return x;
}

template <class TS, bool AKS, bool BKS, class E>
__global__ __launch_bounds__(TS::THREADS, 2) void k_layer_gemm(GemmJob g, E e, int mt, int nt, int splits, int per_split) {
    extern __shared__ __align__(16) unsigned char smem[];
    TilePlace t;
    if (!place_tile(blockIdx.x, mt, nt, splits, t)) return;
    const JobExtent x = job_extent(g);
    const long long m0 = (long long)t.m * TS::BM, n0 = (long long)t.n * TS::BN;
    if (m0 >= x.M) return;
    const int s0 = t.split * per_split, s1 = s0 + per_split < x.stages ? s0 + per_split : x.stages;
    f32x16 acc[TS::MT][TS::NT];
    gemm_tile<TS, AKS, BKS>(acc, g.A, g.B, m0, n0, g.a_rows, g.b_rows, s0, s1, smem);
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, l32 = lane & 31, hb = lane >> 5;
    const int wm = wave / TS::WN, wn = wave % TS::WN;
    typedef typename EpilogueOf<E>::type Store;
#pragma unroll
    for (int j = 0; j < TS::NT; ++j)
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const int n = (int)n0 + (wn * TS::NT + j) * 32 + 16 * p + 8 * hb;
            float b[8];
            Store::bias(e, n, b);
#pragma unroll
            for (int i = 0; i < TS::MT; ++i) {
                const long long m = m0 + (wm * TS::MT + i) * 32 + l32;
                float v[8];
                granule8(acc[i][j], p, v);
                Store::store(e, t.split, m, n, v, b);
            }
        }
}

// The sum of the splits' results, in order, and the epilogue.  One thread per eight columns.
template <class E>
__global__ __launch_bounds__(256) void k_layer_reduce(GemmJob g, E e, const float* __restrict__ slots, int splits, long long Np, long long stride,
                                                      long long total) {
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i >= total) return;
    const long long per = Np / 8, m = i / per;
    const int n = (int)(i - m * per) * 8;
    if (m >= job_extent(g).M) return;
    const float* s = slots + (size_t)m * Np + n;
    f32x4 a = f32x4{0}, b = f32x4{0};
#pragma unroll 4
    for (int k = 0; k < splits; ++k, s += stride) {
        a += *reinterpret_cast<const f32x4*>(s);
        b += *reinterpret_cast<const f32x4*>(s + 4);
    }
    float v[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}, bias[8];
    typedef typename EpilogueOf<E>::type Store;
    Store::bias(e, n, bias);
    Store::store(e, 0, m, n, v, bias);
}

// Scores of a tile and what the softmax needs of them: each row's maximum over the tile's columns, the sum of the exponentials relative to it and, where
// the gradients follow, those exponentials.  They are kept as fp16 scaled by 2^15: 11 bits from 2^-29 of the tile's maximum up, an absolute error of
// 2^-40 of it below, so a probability is off by at most 2^-12 of itself or 2^-40; one exponential per entry serves the statistics and the gradient.
template <class TS, bool KEEP>
__global__ __launch_bounds__(TS::THREADS, 2) void k_ce_scores(GemmJob g, CeEpilogue e, int mt, int nt) {
    extern __shared__ __align__(16) unsigned char smem[];
    TilePlace t;
    if (!place_tile(blockIdx.x, mt, nt, 1, t)) return;
    const JobExtent x = job_extent(g);
    const long long m0 = (long long)t.m * TS::BM, n0 = (long long)t.n * TS::BN;
    if (m0 >= x.M) return;
    f32x16 acc[TS::MT][TS::NT];
    gemm_tile<TS, false, true>(acc, g.A, g.B, m0, n0, g.a_rows, g.b_rows, 0, g.stages, smem);
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, l32 = lane & 31, hb = lane >> 5;
    const int wm = wave / TS::WN, wn = wave % TS::WN;
    float* top = reinterpret_cast<float*>(smem);                  // [WN][BM]
    float* sum = top + TS::WN * TS::BM;                           // [WN][BM]
    // scores; entries beyond the vocabulary are -inf
#pragma unroll
    for (int j = 0; j < TS::NT; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int n = (int)n0 + (wn * TS::NT + j) * 32 + 8 * q + 4 * hb + r;
                const float b = e.bias == nullptr ? 0.0f : e.bias[n < e.V ? n : e.V - 1];
#pragma unroll
                for (int i = 0; i < TS::MT; ++i) acc[i][j][4 * q + r] = n < e.V ? acc[i][j][4 * q + r] + b : RNNT_NEG_INF;
            }
#pragma unroll
    for (int i = 0; i < TS::MT; ++i) {
        const int row = (wm * TS::MT + i) * 32 + l32;
        float m = RNNT_NEG_INF;
#pragma unroll
        for (int j = 0; j < TS::NT; ++j)
#pragma unroll
            for (int q = 0; q < 16; ++q) m = fmaxf(m, acc[i][j][q]);
        m = both_halves_max(m);
        if (hb == 0) top[wn * TS::BM + row] = m;
        // the label's score: the lane that holds its column writes it
        const int y = e.label[m0 + row] - ((int)n0 + wn * TS::NT * 32);
        if (__any((unsigned)y < 32u * TS::NT)) {
            float h = 0.0f;
#pragma unroll
            for (int j = 0; j < TS::NT; ++j)
#pragma unroll
                for (int q = 0; q < 16; ++q) h = y - 4 * hb == 32 * j + 8 * (q >> 2) + (q & 3) ? acc[i][j][q] : h;
            if ((unsigned)y < 32u * TS::NT && ((y >> 2) & 1) == hb) e.label_score[m0 + row] = h;
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < TS::MT; ++i) {
        const int row = (wm * TS::MT + i) * 32 + l32;
        float m = top[row];
#pragma unroll
        for (int w = 1; w < TS::WN; ++w) m = fmaxf(m, top[w * TS::BM + row]);
        const float c = m == RNNT_NEG_INF ? 0.0f : m;             // (a row of -inf: exponentials of zero)
        float s = 0.0f;
#pragma unroll
        for (int j = 0; j < TS::NT; ++j)
#pragma unroll
            for (int q = 0; q < 16; ++q) {
                const float v = __builtin_amdgcn_exp2f(fmaf(acc[i][j][q] - c, LOG2E_F, 15.0f));
                s += v;
                acc[i][j][q] = v;
            }
        s = both_halves_sum(s);
        if (hb == 0) sum[wn * TS::BM + row] = s;
        if constexpr (KEEP) {
            _Float16* dst = (_Float16*)e.kept + (size_t)(m0 + row) * e.pitch + n0 + wn * TS::NT * 32 + 8 * hb;
#pragma unroll
            for (int j = 0; j < TS::NT; ++j)
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    float v[8];
                    granule8(acc[i][j], p, v);
                    f16x8 h;
#pragma unroll
                    for (int k = 0; k < 8; ++k) h[k] = (_Float16)v[k];
                    *reinterpret_cast<f16x8*>(dst + j * 32 + 16 * p) = h;
                }
        }
        if (wn == 0 && hb == 0) e.stats[(size_t)(m0 + row) * e.tiles_n + t.n].x = m;
    }
    __syncthreads();
    for (int row = tid; row < TS::BM; row += TS::THREADS) {
        float s = sum[row];
#pragma unroll
        for (int w = 1; w < TS::WN; ++w) s += sum[w * TS::BM + row];
        e.stats[(size_t)(m0 + row) * e.tiles_n + t.n].y = s;
    }
}

// Kernels ask for more LDS than the default: once per kernel and device.
template <auto KERNEL, class TS, typename... ARGS>
hipError_t launch_tiles(long long tiles, hipStream_t stream, const ARGS&... args) {
    if (tiles > 0x7ffffff0LL) return hipErrorInvalidValue;
    if (tiles <= 0) return hipSuccess;
    static std::atomic<unsigned long long> done{0};               // one per kernel, a bit per device
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    const unsigned long long bit = 1ull << (dev & 63);
    if (!(done.load(std::memory_order_acquire) & bit)) {
        e = hipFuncSetAttribute(reinterpret_cast<const void*>(KERNEL), hipFuncAttributeMaxDynamicSharedMemorySize, (int)TS::SMEM);
        if (e != hipSuccess) return e;
        done.fetch_or(bit, std::memory_order_release);
    }
    KERNEL<<<dim3((unsigned)((tiles + 7) / 8 * 8)), dim3(TS::THREADS), TS::SMEM, stream>>>(args...);
    return hipGetLastError();
}

template <class TS, bool AKS, bool BKS, class E>
hipError_t gemm_of(const GemmJob& g, const GemmPlan& p, float* slots, const E& e, hipStream_t stream) {
    const int mt = (int)((g.M + TS::BM - 1) / TS::BM), nt = (int)((g.N + TS::BN - 1) / TS::BN);
    if (p.splits <= 1) return launch_tiles<&k_layer_gemm<TS, AKS, BKS, E>, TS>((long long)mt * nt, stream, g, e, mt, nt, 1, g.stages);
    const long long Np = (g.N + 7) / 8 * 8, stride = g.M * Np;
    const StoreEpilogue slot{slots, nullptr, nullptr, Np, stride, g.M, (int)Np, false, true};
    hipError_t err = launch_tiles<&k_layer_gemm<TS, AKS, BKS, StoreEpilogue>, TS>((long long)mt * nt * p.splits, stream, g, slot, mt, nt, p.splits,
                                                                                   p.per_split);
    if (err != hipSuccess) return err;
    const long long total = g.M * (Np / 8);
    if ((total + 255) / 256 > 0x7fffffffLL) return hipErrorInvalidValue;
    k_layer_reduce<E><<<dim3((unsigned)((total + 255) / 256)), dim3(256), 0, stream>>>(g, e, slots, p.splits, Np, stride, total);
    return hipGetLastError();
}
template <bool AKS, bool BKS, class E>
hipError_t gemm_of(const GemmJob& g, const GemmPlan& p, float* slots, const E& e, hipStream_t stream) {
    if (g.M <= 0 || g.N <= 0) return hipSuccess;
    return p.tile == 256 ? gemm_of<TileShape<256>, AKS, BKS, E>(g, p, slots, e, stream) : gemm_of<TileShape<128>, AKS, BKS, E>(g, p, slots, e, stream);
}

}  // namespace

// Rounds of the chip (256 compute units; one large tile each, or two small ones) times a round's time, in units of a large tile's stage (about 1.5 us;
// a small one, with its neighbour beside it, 0.7), with five stages' time for a round's start and end; the slots' way to memory and back.
GemmPlan plan_gemm(long long M, long long N, int stages, size_t slot_cap) {
    GemmPlan best{256, 1, stages};
    double least = 1e300;
    for (int tile : {256, 128}) {
        const double tiles = (double)((M + tile - 1) / tile) * (double)((N + tile - 1) / tile);
        const double at_once = tile == 256 ? 256.0 : 512.0, stage = tile == 256 ? 1.0 : 0.7, ends = tile == 256 ? 5.0 : 4.0;
        for (int splits = 1; splits <= 64 && splits <= std::max(1, stages / 2); ++splits) {
            const GemmPlan p{tile, splits, (stages + splits - 1) / splits};
            if ((p.splits - 1) * p.per_split >= stages && splits > 1) continue;      // an empty split
            if (splits > 1 && gemm_slot_bytes(p, M, N) > slot_cap) break;
            const double rounds = std::max(1.0, (double)(long long)((tiles * splits + at_once - 1) / at_once));
            double t = rounds * (p.per_split * stage + ends);
            if (splits > 1) t += 3.0 + (double)gemm_slot_bytes(p, M, N) * 2.0 / 6e6;       // (6 MB per unit)
            if (t < least) {
                least = t;
                best = p;
            }
        }
    }
    return best;
}

hipError_t launch_linear_gemm(const GemmJob& g, const GemmPlan& p, float* slots, const LinearEpilogue& e, hipStream_t stream) {
    return gemm_of<false, true, LinearEpilogue>(g, p, slots, e, stream);
}
hipError_t launch_store_gemm(bool k_slow, const GemmJob& g, const GemmPlan& p, float* slots, const StoreEpilogue& e, hipStream_t stream) {
    return k_slow ? gemm_of<true, true, StoreEpilogue>(g, p, slots, e, stream) : gemm_of<false, false, StoreEpilogue>(g, p, slots, e, stream);
}
hipError_t launch_ce_gemm(const GemmJob& g, int tile, const CeEpilogue& e, hipStream_t stream) {
    if (g.M <= 0) return hipSuccess;
    const int mt = (int)((g.M + tile - 1) / tile), nt = (int)((g.N + tile - 1) / tile);
    typedef TileShape<256> L;
    typedef TileShape<128> S;
    const long long n = (long long)mt * nt;
    if (tile == 256)
        return e.kept != nullptr ? launch_tiles<&k_ce_scores<L, true>, L>(n, stream, g, e, mt, nt)
                                 : launch_tiles<&k_ce_scores<L, false>, L>(n, stream, g, e, mt, nt);
    return e.kept != nullptr ? launch_tiles<&k_ce_scores<S, true>, S>(n, stream, g, e, mt, nt)
                             : launch_tiles<&k_ce_scores<S, false>, S>(n, stream, g, e, mt, nt);
}

}  // namespace rnnt
