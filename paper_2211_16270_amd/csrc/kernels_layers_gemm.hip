// bf16 matrix products of the linear layer (y, dx, dW) and of the output layer's cross entropy (scores with their statistics; dx, dW).
#include <algorithm>
#include <atomic>
#include <cmath>

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
            const long long s = (n + GK - 1) / GK * g.per_block;
            x.stages = s < x.stages ? (int)s : x.stages;
        }
    }
    return x;
}

template <class TS, bool AKS, bool BKS, Passes HOW, class E>
__device__ __forceinline__ void gemm_workgroup(const GemmJob& g, const E& e, int L, int mt, int nt, int splits, int per_split, unsigned char* smem) {
    TilePlace t;
    if (!place_tile(L, mt, nt, splits, t)) return;
    const JobExtent x = job_extent(g);
    const long long m0 = (long long)t.m * TS::BM, n0 = (long long)t.n * TS::BN;
    if (m0 >= x.M) return;
    const int s0 = t.split * per_split, s1 = s0 + per_split < x.stages ? s0 + per_split : x.stages;
    f32x16 acc[TS::MT][TS::NT];
    constexpr bool LINEAR = std::is_base_of_v<LinearEpilogue, E>;
    // (scores in fp32 are the only other results with a bias)
    if constexpr (LINEAR || (HOW == IN_PARTS && !AKS && BKS))
        gemm_tile<TS, AKS, BKS, HOW>(acc, g.A, g.B, m0, n0, g.a_rows, g.b_rows, s0, s1, smem, ColumnBias{e.bias, e.N, 0.0f});
    else gemm_tile<TS, AKS, BKS, HOW>(acc, g.A, g.B, m0, n0, g.a_rows, g.b_rows, s0, s1, smem, NoBias{});
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int wm = wave / TS::WN, wn = wave % TS::WN, n = (int)n0 + wn * TS::NT * 32 + 8 * (lane & 7);
    unsigned char* area = smem + wave * TURN32_BYTES;
    static_assert(TS::NT == 2 && TS::WAVES * TURN32_BYTES <= TS::SMEM, "a wave's 64 columns");
    typedef typename EpilogueOf<E>::type Store;
    const float factor = Store::factor(e);
    // One loop over the pieces of eight rows; what four of them need of memory is sent for at once (one at a time, three ahead: a residual took 20 us of 16000 x
    // 1024 x 4096, now 10: a wait for such a load is one for the stores in front of it too).
    const long long first = m0 + wm * TS::MT * 32 + (lane >> 3);
    typename Store::Extra mem[4];
#pragma unroll 1
    for (int k = 0; k < 4 * TS::MT; ++k) {
        if (k % 4 == 0) {
#pragma unroll
            for (int q = 0; q < 4; ++q) mem[q] = Store::fetch(e, first + 8 * (k + q), n);
            turn_fence();
            static_for<0, TS::MT>([&](auto i) {
                if (k / 4 == decltype(i)::value) {
                    turn32_put(area, 0, acc[decltype(i)::value][0], lane);
                    turn32_put(area, 1, acc[decltype(i)::value][1], lane);
                }
            });
            turn_fence();
        }
        float v[8];
        turn32_take(area, k % 4, lane, v);
        // (a register array indexed by the loop's counter would lie in memory)
        const typename Store::Extra r = k & 2 ? (k & 1 ? mem[3] : mem[2]) : (k & 1 ? mem[1] : mem[0]);
        Store::store(e, first + 8 * k, n, v, r, factor, t.split);
    }
}

// A product and how its workgroups are dealt out
template <class E>
struct TileJob {
    GemmJob g;
    E e;
    int mt, nt, splits, per_split;
    __host__ __device__ long long workgroups() const { return ((long long)mt * nt * splits + 7) / 8 * 8; }
};
// y, or a split of it.  Bound by the matrix units' power in long sums, by each tile's start and epilogue in short ones: 16000 x 1024 x 4096 143 to 147 us (930
// TFLOP/s) plain, 160 with silu, 177 with gelu, 208 to 212 with gelu, dropout and the saved z (their vector work and its bytes, nothing hides them); 8000 x 512 x 2048
// 28 plain, 39 with silu, dropout and the saved z.
template <class TS, bool AKS, bool BKS, Passes HOW, class E>
__global__ __launch_bounds__(TS::THREADS, 2) void k_layer_gemm(TileJob<E> j) {
    extern __shared__ __align__(16) unsigned char smem[];
    if (blockIdx.x == 0) pass_rng(j.e);
    gemm_workgroup<TS, AKS, BKS, HOW, E>(j.g, j.e, blockIdx.x, j.mt, j.nt, j.splits, j.per_split, smem);
}
// dx and dW; the product whose workgroups take longer goes first (16000 x 1024 x 4096: 225 to 240 us, behind the other 308).  Bound like k_layer_gemm: CE, 9288 x
// 1024 x 32768, 1190 us (1050 TFLOP/s; workgroups of 145 and 512 stages leave a tenth of the compute units' time unused).
template <class TS, Passes HOW>
__global__ __launch_bounds__(TS::THREADS, 2) void k_layer_grads(TileJob<StoreEpilogue> x, TileJob<StoreEpilogue> w, int wgs_x, int wgs_w) {
    extern __shared__ __align__(16) unsigned char smem[];
    const bool x_first = x.per_split > w.per_split;
    const int L = blockIdx.x, is_x = x_first ? L < wgs_x : L >= wgs_w;
    if (is_x) gemm_workgroup<TS, false, false, HOW, StoreEpilogue>(x.g, x.e, x_first ? L : L - wgs_w, x.mt, x.nt, x.splits, x.per_split, smem);
    else gemm_workgroup<TS, true, true, HOW, StoreEpilogue>(w.g, w.e, x_first ? L - wgs_x : L, w.mt, w.nt, w.splits, w.per_split, smem);
}

// The sum of the splits' results, in order, and the epilogue.  One thread per eight columns.  Bound by its bytes and, at 4 to 12 us, by the launch.
template <class E>
struct ReduceJob {
    GemmJob g;
    E e;
    const float* slots;
    int splits;
    long long Np, stride, total;
    __host__ __device__ unsigned workgroups() const { return splits > 1 ? (unsigned)((total + 255) / 256) : 0u; }
};
template <class E>
__device__ __forceinline__ void reduce_workgroup(const ReduceJob<E>& r, unsigned block) {
    const long long i = (long long)block * 256 + threadIdx.x;
    if (i >= r.total) return;
    const long long per = r.Np / 8, m = i / per;
    const int n = (int)(i - m * per) * 8;
    if (m >= job_extent(r.g).M) return;
    typedef typename EpilogueOf<E>::type Store;
    const typename Store::Extra x = Store::fetch(r.e, m, n);
    const float* s = r.slots + (size_t)m * r.Np + n;
    f32x4 a = f32x4{0}, b = f32x4{0};
#pragma unroll 4
    for (int k = 0; k < r.splits; ++k, s += r.stride) {
        a += *reinterpret_cast<const f32x4*>(s);
        b += *reinterpret_cast<const f32x4*>(s + 4);
    }
    float v[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}, bias[8];
    Store::bias(r.e, n, bias);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] += bias[k];
    Store::store(r.e, m, n, v, x, Store::factor(r.e));
}
template <class E>
__global__ __launch_bounds__(256) void k_layer_reduce(ReduceJob<E> r) {
    if (blockIdx.x == 0) pass_rng(r.e);
    reduce_workgroup(r, blockIdx.x);
}
__global__ __launch_bounds__(256) void k_layer_reduce_grads(ReduceJob<StoreEpilogue> x, ReduceJob<StoreEpilogue> w, SumJob db, int db_blocks, int db_rows) {
    __shared__ float red[8][32];
    unsigned L = blockIdx.x;
    if (L < x.workgroups()) return reduce_workgroup(x, L);
    L -= x.workgroups();
    if (L < w.workgroups()) return reduce_workgroup(w, L);
    sum_parts(db, db_blocks, db_rows, (int)(L - w.workgroups()), red);
}

// Scores of a tile and what the softmax needs of them: each row's maximum over the tile's columns, the sum of the exponentials relative to it and, where
// the gradients follow, those exponentials.  They are kept as fp16 scaled by 2^15: 11 bits from 2^-29 of the tile's maximum up, an absolute error of
// 2^-40 of it below, so a probability is off by at most 2^-12 of itself or 2^-40; one exponential per entry serves the statistics and the gradient.  Bound by the
// products and, behind each tile's, by its exponentials: 9288 x 1024 x 32768 700 to 735 us (870 TFLOP/s, 16 stages a tile).
template <class TS, bool KEEP>
__global__ __launch_bounds__(TS::THREADS, 2) void k_ce_scores(GemmJob g, CeEpilogue e, int mt, int nt) {
    extern __shared__ __align__(16) unsigned char smem[];
    TilePlace t;
    if (!place_tile(blockIdx.x, mt, nt, 1, t)) return;
    const JobExtent x = job_extent(g);
    const long long m0 = (long long)t.m * TS::BM, n0 = (long long)t.n * TS::BN;
    if (m0 >= x.M) return;
    f32x16 acc[TS::MT][TS::NT];
    // (entries beyond the vocabulary are -inf)
    gemm_tile<TS, false, true, ONCE>(acc, g.A, g.B, m0, n0, g.a_rows, g.b_rows, 0, g.stages, smem, ColumnBias{e.bias, e.V, RNNT_NEG_INF});
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, l32 = lane & 31, hb = lane >> 5;
    const int wm = wave / TS::WN, wn = wave % TS::WN;
    float* top = reinterpret_cast<float*>(smem);                  // [WN][BM]
    float* sum = top + TS::WN * TS::BM;                           // [WN][BM]
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
            unsigned char* area = smem + 2 * TS::WN * TS::BM * 4 + wave * TURN_BYTES;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float v[8];
                granule8(acc[i][k >> 1], k & 1, v);
                f16x8 h;
#pragma unroll
                for (int x = 0; x < 8; ++x) h[x] = (_Float16)v[x];
                turn_put(area, k >> 1, k & 1, lane, __builtin_bit_cast(u32x4, h));
            }
            turn_fence();
#pragma unroll
            for (int k = 0; k < 4; ++k)
                *reinterpret_cast<u32x4*>((_Float16*)e.kept + (size_t)(m0 + (wm * TS::MT + i) * 32 + 8 * k + (lane >> 3)) * e.pitch + n0 +
                                          wn * TS::NT * 32 + 8 * (lane & 7)) = turn_take(area, k, lane);
            turn_fence();
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

template <class TS, class E>
TileJob<E> tile_job(const GemmJob& g, const E& e, int splits, int per_split) {
    return TileJob<E>{g, e, (int)((g.M + TS::BM - 1) / TS::BM), (int)((g.N + TS::BN - 1) / TS::BN), splits, per_split};
}
inline long long padded8(long long n) { return (n + 7) / 8 * 8; }
StoreEpilogue slot_epilogue(const GemmJob& g, float* slots) {
    return StoreEpilogue{slots, nullptr, 1.0f, nullptr, nullptr, padded8(g.N), g.M * padded8(g.N), Bias{}, g.M, (int)padded8(g.N), false};
}
template <class E>
ReduceJob<E> reduce_job(const GemmJob& g, const E& e, const float* slots, int splits) {
    return ReduceJob<E>{g, e, slots, splits, padded8(g.N), g.M * padded8(g.N), g.M * (padded8(g.N) / 8)};
}

template <class TS, Passes HOW, class E>
hipError_t gemm_of(const GemmJob& g, const GemmPlan& p, float* slots, const E& e, hipStream_t stream) {
    if (p.splits <= 1) {
        const TileJob<E> j = tile_job<TS>(g, e, 1, g.stages);
        return launch_tiles<&k_layer_gemm<TS, false, true, HOW, E>, TS>(j.workgroups(), stream, j);
    }
    const TileJob<StoreEpilogue> j = tile_job<TS>(g, slot_epilogue(g, slots), p.splits, p.per_split);
    hipError_t err = launch_tiles<&k_layer_gemm<TS, false, true, HOW, StoreEpilogue>, TS>(j.workgroups(), stream, j);
    if (err != hipSuccess) return err;
    const ReduceJob<E> r = reduce_job(g, e, slots, p.splits);
    if ((r.total + 255) / 256 > 0x7fffffffLL) return hipErrorInvalidValue;
    k_layer_reduce<E><<<dim3(r.workgroups()), dim3(256), 0, stream>>>(r);
    return hipGetLastError();
}
template <Passes HOW, class E>
hipError_t gemm_of(const GemmJob& g, const GemmPlan& p, float* slots, const E& e, hipStream_t stream) {
    if (g.M <= 0 || g.N <= 0) return hipSuccess;
    return p.tile == 256 ? gemm_of<TileShape<256>, HOW>(g, p, slots, e, stream) : gemm_of<TileShape<128>, HOW>(g, p, slots, e, stream);
}

template <class TS, Passes HOW>
hipError_t grad_gemms(const GradGemm& dx, const GradGemm& dw, hipStream_t stream) {
    TileJob<StoreEpilogue> x{}, w{};
    if (dx.g.M > 0) x = tile_job<TS>(dx.g, dx.splits > 1 ? slot_epilogue(dx.g, dx.slots) : dx.e, dx.splits, dx.splits > 1 ? dx.per_split : dx.g.stages);
    if (dw.g.M > 0) w = tile_job<TS>(dw.g, dw.splits > 1 ? slot_epilogue(dw.g, dw.slots) : dw.e, dw.splits, dw.splits > 1 ? dw.per_split : dw.g.stages);
    const long long nx = x.workgroups(), nw = w.workgroups();
    if (nx + nw > 0x7ffffff0LL) return hipErrorInvalidValue;
    return launch_tiles<&k_layer_grads<TS, HOW>, TS>(nx + nw, stream, x, w, (int)nx, (int)nw);
}

}  // namespace

// Rounds of the chip (256 compute units; one large tile each, or two small ones) times a round's time, in units of a large tile's stage (about 1.5 us;
// a small one, with its neighbour beside it, 0.7), with some stages' time for a round's start and end: in a product by itself nine, of which a small tile's neighbour
// hides a part; where two products share a launch, less.  Small tiles follow each other as places get free, so they go by parts of rounds (0.3 for the last):
// 12000 x 512 x 1536, 2.2 rounds of small tiles 39.7 us and with silu, dropout and the saved z 51.8, two of large ones 44.2 and 65.6; 10000 x 640 x 2560, 3.1 and 2:
// 58.2 and 75.5, 52.1 and 74.7.  Then the slots' way to memory and back.
namespace {
constexpr double STAGE_TIME[2] = {1.0, 0.7}, ENDS_TIME[2] = {5.0, 4.0}, ALONE_ENDS[2] = {9.0, 5.5}, AT_ONCE[2] = {256.0, 512.0}, BYTES_PER_UNIT = 6e6, LAUNCH_TIME = 3.0;
constexpr int SPLITS[] = {1, 2, 3, 4, 5, 6, 7, 8, 10, 12, 14, 16, 20, 24, 32, 48, 64}, N_SPLITS = sizeof(SPLITS) / sizeof(int);
struct Choice {
    GemmPlan p;
    double workgroups, time, extra;      // number, each one's time, the slots' time
};
// The splits of a product with tiles of shape k that are possible
int choices(int k, long long M, long long N, int stages, size_t slot_cap, double ends, Choice (&c)[N_SPLITS]) {
    const int tile = k == 0 ? 256 : 128;
    const double tiles = (double)((M + tile - 1) / tile) * (double)((N + tile - 1) / tile);
    int n = 0;
    for (int splits : SPLITS) {
        const GemmPlan p{tile, splits, (stages + splits - 1) / splits};
        const size_t bytes = gemm_slot_bytes(p, M, N);
        if (splits > 1 && (splits > stages / 2 || (splits - 1) * p.per_split >= stages || bytes > slot_cap)) continue;
        c[n++] = Choice{p, tiles * splits, p.per_split * STAGE_TIME[k] + ends, (double)bytes * 2.0 / BYTES_PER_UNIT};
    }
    return n;
}
}  // namespace
GemmPlan plan_gemm(long long M, long long N, int stages, size_t slot_cap) {
    GemmPlan best{256, 1, stages};
    double least = 1e300;
    for (int k = 0; k < 2; ++k) {
        Choice c[N_SPLITS];
        const int n = choices(k, M, N, stages, slot_cap, ALONE_ENDS[k], c);
        for (int i = 0; i < n; ++i) {
            const double part = c[i].workgroups / AT_ONCE[k], rounds = std::max(1.0, k == 0 ? std::ceil(part) : part + 0.3);
            const double t = rounds * c[i].time + (c[i].p.splits > 1 ? LAUNCH_TIME + c[i].extra : 0.0);
            if (t < least) {
                least = t;
                best = c[i].p;
            }
        }
    }
    return best;
}
// The same for two products that share a launch: workgroups of both fill the chip one after the other.
PairPlan plan_pair(long long Mx, long long Nx, int stages_x, long long Mw, long long Nw, int stages_w, size_t slot_cap, bool small) {
    PairPlan best{256, {256, 1, stages_x}, {256, 1, stages_w}};
    double least = 1e300;
    for (int k = small ? 1 : 0; k < 2; ++k) {
        Choice x[N_SPLITS], w[N_SPLITS];
        const int nx = choices(k, Mx, Nx, stages_x, slot_cap, ENDS_TIME[k], x), nw = choices(k, Mw, Nw, stages_w, slot_cap, ENDS_TIME[k], w);
        for (int i = 0; i < nx; ++i)
            for (int j = 0; j < nw; ++j) {
                // at least one workgroup's time; the last round is on average half empty
                const double work = (x[i].workgroups * x[i].time + w[j].workgroups * w[j].time) / AT_ONCE[k];
                const double longest = std::max(x[i].workgroups > 0 ? x[i].time : 0.0, w[j].time), shortest = std::min(x[i].time, w[j].time);
                double t = work > longest ? work + 0.5 * shortest : longest;
                if (x[i].p.splits > 1 || w[j].p.splits > 1) t += LAUNCH_TIME + x[i].extra + w[j].extra;
                if (t < least) {
                    least = t;
                    best = PairPlan{k == 0 ? 256 : 128, x[i].p, w[j].p};
                }
            }
    }
    return best;
}

hipError_t launch_linear_gemm(const GemmJob& g, const GemmPlan& p, float* slots, const LinearEpilogue& e, hipStream_t stream) {
    return gemm_of<ONCE>(g, p, slots, e, stream);
}
hipError_t launch_linear_gemm(const GemmJob& g, const GemmPlan& p, float* slots, const LinearEpilogue32& e, hipStream_t stream) {
    return gemm_of<IN_PARTS>(g, p, slots, e, stream);
}
hipError_t launch_scores_f32(const GemmJob& g, int tile, const StoreEpilogue& e, hipStream_t stream) {
    return gemm_of<IN_PARTS>(g, GemmPlan{tile, 1, g.stages}, nullptr, e, stream);
}
hipError_t launch_linear_reduce(bool f32, long long M, int N, int splits, const float* slots, const LinearEpilogue& e, hipStream_t stream) {
    GemmJob g{};
    g.M = M;
    g.N = N;
    const ReduceJob<LinearEpilogue> r = reduce_job(g, e, slots, splits);
    if (f32) {
        const ReduceJob<LinearEpilogue32> q = reduce_job(g, LinearEpilogue32{e}, slots, splits);
        k_layer_reduce<LinearEpilogue32><<<dim3(q.workgroups()), dim3(256), 0, stream>>>(q);
    } else k_layer_reduce<LinearEpilogue><<<dim3(r.workgroups()), dim3(256), 0, stream>>>(r);
    return hipGetLastError();
}
hipError_t launch_grad_gemms(bool parts, int tile, const GradGemm& dx, const GradGemm& dw, const SumJob& db, hipStream_t stream) {
    if (dx.g.M > 0 || dw.g.M > 0) {
        typedef TileShape<256> L;
        typedef TileShape<128> S;
        const bool twice = dx.g.A.wrap > 0 || dw.g.B.wrap > 0;
        if (twice && tile != 128) return hipErrorInvalidValue;          // (planned for another kernel)
        const hipError_t e = parts   ? (tile == 256 ? grad_gemms<L, IN_PARTS>(dx, dw, stream) : grad_gemms<S, IN_PARTS>(dx, dw, stream))
                             : twice ? grad_gemms<S, TWICE>(dx, dw, stream)
                                     : (tile == 256 ? grad_gemms<L, ONCE>(dx, dw, stream) : grad_gemms<S, ONCE>(dx, dw, stream));
        if (e != hipSuccess) return e;
    }
    ReduceJob<StoreEpilogue> x{}, w{};
    if (dx.g.M > 0) x = reduce_job(dx.g, dx.e, dx.slots, dx.splits);
    if (dw.g.M > 0) w = reduce_job(dw.g, dw.e, dw.slots, dw.splits);
    const long long n = (long long)x.workgroups() + w.workgroups() + (db.out != nullptr ? (db.N + 31) / 32 : 0);
    if (n == 0) return hipSuccess;
    if (n > 0x7fffffffLL) return hipErrorInvalidValue;
    k_layer_reduce_grads<<<dim3((unsigned)n), dim3(256), 0, stream>>>(x, w, db, (int)sum_blocks(db.rows, db.N), sum_rows(db.rows, db.N));
    return hipGetLastError();
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
