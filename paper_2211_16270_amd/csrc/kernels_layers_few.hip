// A few rows (at most 64) through a layer: single tokens, beams.  The product is bound by reading W, the call by latency, so one launch does it all
// (1 row, K = 640, N = 2560: 4.4 us, W's 3.3 MB at a copy's rate 0.7).  Times in this file: a call among others in a captured graph; the profiler shows 0.6 to 0.8 more.
#include <algorithm>

#include "layers_device.h"

namespace rnnt {

namespace {

typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef short s16x8_t __attribute__((ext_vector_type(8)));
constexpr int FW = 8;              // waves of a workgroup: each takes every eighth step of 32 along k
constexpr int FC = 32;             // columns of a workgroup: 64 bytes of a row of W
constexpr int FD = 4;              // steps whose loads are in flight

// Eight values of a row as they lie there, zeros from `live` on
__device__ __forceinline__ bf16x8 raw8(const bf16_t* p, int live) {
    if (live >= 8) return *reinterpret_cast<const bf16x8_any*>(p);
    s16x8_t v = s16x8_t{0};
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < live) v[j] = reinterpret_cast<const short*>(p)[j];
    return __builtin_bit_cast(bf16x8, v);
}

template <class STORE>
struct FewLinear {
    LinearEpilogue e;
    __device__ __forceinline__ void first() const { pass_rng(e); }
    // columns n .. n + 7 (granule g of the workgroup's 32) of row m
    __device__ __forceinline__ void operator()(int m, int n, int, float (&v)[8]) const {
        float b[8];
        STORE::bias(e, n, b);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] += b[k];
        STORE::store(e, m, n, v, STORE::fetch(e, m, n));
    }
};
// Statistics of the 32 columns of a row (four neighbouring lanes hold them), as k_ce_scores leaves them for its tiles
struct FewCe {
    CeEpilogue e;
    __device__ __forceinline__ void first() const {}
    __device__ __forceinline__ void operator()(int m, int n, int block, float (&v)[8]) const {
        float b[8];
        load_bias8(e.bias, n < e.V ? n : e.V - 1, e.V, b);
        const int y = e.label[m] - n;
        float top = RNNT_NEG_INF;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[j] = n + j < e.V ? v[j] + b[j] : RNNT_NEG_INF;
            top = fmaxf(top, v[j]);
            if (y == j && n + j < e.V) e.label_score[m] = v[j];
        }
        top = fmaxf(top, __shfl_xor(top, 1, 64));
        top = fmaxf(top, __shfl_xor(top, 2, 64));
        const float c = top == RNNT_NEG_INF ? 0.0f : top;
        float s = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[j] = __builtin_amdgcn_exp2f(fmaf(v[j] - c, LOG2E_F, 15.0f));
            s += v[j];
        }
        s += __shfl_xor(s, 1, 64);
        s += __shfl_xor(s, 2, 64);
        if (n % FC == 0) e.stats[(size_t)m * e.tiles_n + block] = make_float2(top, s);
        if (e.kept != nullptr) store8((_Float16*)e.kept + (size_t)m * e.pitch + n, 8, v);
    }
};

// The eight waves' sums -> the epilogue, or this split's slot
template <int MT, class E>
__device__ __forceinline__ void few_finish(const FewJob& j, const E& e, const f32x4 (&acc)[MT][2], unsigned char* smem, float* __restrict__ slots, int block,
                                           int m0, int n0) {
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    __syncthreads();
    // register r of lane l: column 4 (l / 16) + r of its 16, row l % 16
    float* part = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int c = 0; c < 2; ++c)
            *reinterpret_cast<f32x4*>(part + ((wave * MT + i) * 16 + (lane & 15)) * FC + c * 16 + 4 * (lane >> 4)) = acc[i][c];
    __syncthreads();
    if (tid < MT * 64) {
        const int in = tid >> 2, m = m0 + in, g = tid & 3;
        f32x4 p = f32x4{0}, q = f32x4{0};
#pragma unroll
        for (int k = 0; k < FW; ++k) {
            const float* s = part + ((size_t)k * MT * 16 + in) * FC + g * 8;
            p += *reinterpret_cast<const f32x4*>(s);
            q += *reinterpret_cast<const f32x4*>(s + 4);
        }
        float v[8] = {p[0], p[1], p[2], p[3], q[0], q[1], q[2], q[3]};
        if (m >= j.M) return;
        if (slots == nullptr) e(m, n0 + g * 8, block, v);
        else {
            const int Np = (j.N + 7) / 8 * 8;
            if (n0 + g * 8 < Np) store8(slots + ((size_t)blockIdx.y * j.M + m) * Np + n0 + g * 8, 8, v);
        }
    }
}

// rows x 32 columns of x W per workgroup, MT blocks of 16 rows.  A wave brings its steps (32 of k) of W through registers into LDS of its own, where the
// transposing read makes MFMA fragments of them; x comes as fragments from memory.  The eight waves' sums meet in LDS.  Neighbouring column blocks share
// lines of W: they go to one XCD.  What bounds it: latency (the launch, two trips to memory, the reduction).
// WHOLE: K and N are multiples of 32, no piece has an end in it (the code for ends, eight loads under eight conditions for each load, takes longer to fetch
// than to run).
// Rows in several workgroups: gridDim.z.  A long sum is split over workgroups too (gridDim.y > 1), whose results go to slots [split][M][N up to 8].
template <int MT, bool WHOLE, class E>
__global__ __launch_bounds__(64 * FW) void k_few_rows(FewJob j, E e, int blocks, float* __restrict__ slots, int per_split) {
    __shared__ __align__(16) unsigned char smem[FW * MT * 16 * FC * 4];
    static_assert(MT * 16 * FC * 4 >= 2048, "a step of W per wave");
    const int per = (blocks + 7) >> 3, block = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per || block >= blocks) return;
    const int m0 = blockIdx.z * MT * 16;
    if (block == 0 && m0 == 0 && slots == nullptr) e.first();
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, n0 = block * FC;
    const int K = j.K, N = j.N;
    unsigned char* area = smem + wave * 2048;
    const bf16_t* W = (const bf16_t*)j.W + n0 + (lane & 3) * 8;
    const int wk = lane >> 2, wlive = N - n0 - (lane & 3) * 8, xk = 8 * (lane >> 4);
    const bf16_t* x[MT];
    bool row_ok[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int row = m0 + 16 * i + (lane & 15);
        row_ok[i] = row < j.M;
        x[i] = (const bf16_t*)j.x + (size_t)(row_ok[i] ? row : 0) * K;
    }
    f32x4 acc[MT][2];
#pragma unroll
    for (int i = 0; i < MT; ++i) acc[i][0] = acc[i][1] = f32x4{0};
    bf16x8 w[FD][2], a[FD][MT];
    auto fetch = [&](auto slot_tag, int k0) {
        constexpr int s = decltype(slot_tag)::value;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int k = k0 + 16 * u + wk;
            if constexpr (WHOLE) w[s][u] = *reinterpret_cast<const bf16x8*>(W + (size_t)(k < K ? k : 0) * N);
            else w[s][u] = raw8(W + (size_t)(k < K ? k : 0) * N, k < K ? wlive : 0);
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const bf16_t* p = x[i] + (k0 + xk < K ? k0 + xk : 0);
            if constexpr (WHOLE) a[s][i] = *reinterpret_cast<const bf16x8*>(p);
            else a[s][i] = raw8(p, row_ok[i] ? K - (k0 + xk) : 0);
        }
    };
    const int fj = (lane >> 2) & 3, fc = lane & 3, fg = lane >> 4;
    auto step = [&](auto slot_tag) {
        constexpr int s = decltype(slot_tag)::value;
#pragma unroll
        for (int u = 0; u < 2; ++u) *reinterpret_cast<bf16x8*>(area + (16 * u + wk) * 64 + (lane & 3) * 16) = w[s][u];
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        bf16x8 f[2];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            // lane 16 g + 4 j + c supplies columns 4 c .. of row 8 g + j (+ 4); lane i of the 16 receives rows 8 g .. + 7 of column i
            const unsigned char* p = area + (8 * fg + fj) * 64 + c * 32 + fc * 8;
            const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(p));
            const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(p + 4 * 64));
            const s16x8_t v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            f[c] = __builtin_bit_cast(bf16x8, v);
        }
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int c = 0; c < 2; ++c) acc[i][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[c], a[s][i], acc[i][c], 0, 0, 0);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    };
    const int all = (K + 31) / 32, first = blockIdx.y * per_split, steps = first + per_split < all ? first + per_split : all;
    static_for<0, FD>([&](auto s) {
        const int t = first + wave + FW * decltype(s)::value;
        if (t < steps) fetch(s, 32 * t);
    });
    for (int t = first + wave; t < steps; t += FW * FD)
        static_for<0, FD>([&](auto s) {
            constexpr int q = decltype(s)::value;
            if (t + FW * q < steps) {
                step(s);
                if (t + FW * (q + FD) < steps) fetch(s, 32 * (t + FW * (q + FD)));
            }
        });
    few_finish<MT>(j, e, acc, smem, slots, block, m0, n0);
}

// The same in fp32 on the fp32 matrix instruction (16 x 16 x 4), which takes its operands as they lie: a wave's step of 32 along k is eight of them, the
// i-th with k = 8 g + i in the lanes of group g = l / 16, so that a lane's eight values of x are one piece.  1 x 640 x 2560 6.3 us, 64 x 640 x 2560 9.8: sixteen loads of four bytes of W a
// step, two steps of them in flight.
template <int MT, bool WHOLE, class E>
__global__ __launch_bounds__(64 * FW) void k_few_rows_f32(FewJob j, E e, int blocks, float* __restrict__ slots, int per_split) {
    __shared__ __align__(16) unsigned char smem[FW * MT * 16 * FC * 4];
    const int per = (blocks + 7) >> 3, block = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per || block >= blocks) return;
    const int m0 = blockIdx.z * MT * 16;
    if (block == 0 && m0 == 0 && slots == nullptr) e.first();
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, n0 = block * FC, g = lane >> 4, l16 = lane & 15;
    const int K = j.K, N = j.N;
    const float* W = (const float*)j.W;
    const float* x[MT];
    bool row_ok[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int row = m0 + 16 * i + l16;
        row_ok[i] = row < j.M;
        x[i] = (const float*)j.x + (size_t)(row_ok[i] ? row : 0) * K;
    }
    f32x4 acc[MT][2];
#pragma unroll
    for (int i = 0; i < MT; ++i) acc[i][0] = acc[i][1] = f32x4{0};
    constexpr int D = MT == 4 ? 1 : 2;                            // steps in flight
    float w[D][2][8], a[D][MT][8];
    auto fetch = [&](auto slot_tag, int k0) {
        constexpr int s = decltype(slot_tag)::value;
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int k = k0 + 8 * g + i, n = n0 + 16 * c + l16;
                const bool ok = k < K && (WHOLE || n < N);
                const float v = W[ok ? (size_t)k * N + n : 0];
                w[s][c][i] = ok ? v : 0.0f;
            }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int k = k0 + 8 * g;
            load8(x[i] + (k < K ? k : 0), WHOLE ? 8 : row_ok[i] ? (K - k < 0 ? 0 : K - k) : 0, a[s][i]);
        }
    };
    auto step = [&](auto slot_tag) {
        constexpr int s = decltype(slot_tag)::value;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int c = 0; c < 2; ++c) acc[m][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(w[s][c][i], a[s][m][i], acc[m][c], 0, 0, 0);
    };
    const int all = (K + 31) / 32, first = blockIdx.y * per_split, steps = first + per_split < all ? first + per_split : all;
    static_for<0, D>([&](auto s) {
        const int t = first + wave + FW * decltype(s)::value;
        if (t < steps) fetch(s, 32 * t);
    });
    for (int t = first + wave; t < steps; t += FW * D)
        static_for<0, D>([&](auto s) {
            constexpr int q = decltype(s)::value;
            if (t + FW * q < steps) {
                step(s);
                if (t + FW * (q + D) < steps) fetch(s, 32 * (t + FW * (q + D)));
            }
        });
    few_finish<MT>(j, e, acc, smem, slots, block, m0, n0);
}

// Blocks of 16 rows per workgroup: as few as leave a workgroup per compute unit at most.  A wave's loads of x are what takes long, and W comes from the L2 for
// all but the first (bf16, 64 rows, K = 640, N = 2560: 5.6 us, 7.6 with all rows in one workgroup; K = 2560, N = 640 7.2 and 14.9; fp32 9.8 and 16.2, but 15.5 and
// 13.2, where the long sum is split too).
int few_blocks(int M, int N) {
    const int columns = (N + FC - 1) / FC, all = (M + 15) / 16;
    int mt = 1;
    while (mt < 4 && mt < all && columns * ((all + mt - 1) / mt) > 256) mt *= 2;
    return mt;
}
template <bool F32, class E>
hipError_t launch_few(const FewJob& j, const E& e, int splits, float* slots, hipStream_t stream) {
    if (j.M <= 0 || j.M > FEW_ROWS) return j.M <= 0 ? hipSuccess : hipErrorInvalidValue;
    const int blocks = (j.N + FC - 1) / FC, per = ((j.K + 31) / 32 + splits - 1) / splits;
    const int mt = few_blocks(j.M, j.N);
    const dim3 grid((unsigned)((blocks + 7) / 8 * 8), (unsigned)splits, (unsigned)((j.M + 16 * mt - 1) / (16 * mt)));
    const bool whole = j.K % 32 == 0 && j.N % FC == 0;
    auto go = [&](auto mt) {
        constexpr int MT = decltype(mt)::value;
        if constexpr (F32) {
            if (whole) k_few_rows_f32<MT, true, E><<<grid, dim3(64 * FW), 0, stream>>>(j, e, blocks, slots, per);
            else k_few_rows_f32<MT, false, E><<<grid, dim3(64 * FW), 0, stream>>>(j, e, blocks, slots, per);
        } else if (whole) k_few_rows<MT, true, E><<<grid, dim3(64 * FW), 0, stream>>>(j, e, blocks, slots, per);
        else k_few_rows<MT, false, E><<<grid, dim3(64 * FW), 0, stream>>>(j, e, blocks, slots, per);
        return hipGetLastError();
    };
    return mt == 1 ? go(std::integral_constant<int, 1>{}) : mt == 2 ? go(std::integral_constant<int, 2>{}) : go(std::integral_constant<int, 4>{});
}

}  // namespace

// Long sums are shared by as many workgroups as fill the chip, each with a step per wave at least: in fp32, whose steps take sixteen loads of W each, from five
// steps per wave on (1 row, K = 2560, N = 640: 7.5 us, 14.7 in one workgroup per 32 columns; 64 rows 15.5 and 16.4), in bf16 from seventeen (with ten, split, 6.8 us
// and 9.4 for 64 rows; 5.9 and 7.2 so: the second launch takes what the split saves).
int few_splits(bool f32, long long M, int K, int N) {
    if (M < 1 || M > FEW_ROWS) return 1;
    const int steps = (K + 31) / 32, mt = few_blocks((int)M, N), blocks = (N + FC - 1) / FC * (((int)M + 16 * mt - 1) / (16 * mt));
    if (steps <= (f32 ? 4 : 16) * FW) return 1;
    const int most = std::min(steps / FW, std::max(1, 256 / blocks)), per = (steps + most - 1) / most;
    return (steps + per - 1) / per;
}
hipError_t launch_few_linear(const FewJob& j, int splits, float* slots, const LinearEpilogue& e, hipStream_t stream) {
    const hipError_t err = j.f32 ? launch_few<true>(j, FewLinear<LinearStore32>{e}, splits, splits > 1 ? slots : nullptr, stream)
                                 : launch_few<false>(j, FewLinear<LinearStore>{e}, splits, splits > 1 ? slots : nullptr, stream);
    return err != hipSuccess || splits <= 1 ? err : launch_linear_reduce(j.f32, j.M, j.N, splits, slots, e, stream);
}
hipError_t launch_few_ce(const FewJob& j, const CeEpilogue& e, hipStream_t stream) {
    return j.f32 ? launch_few<true>(j, FewCe{e}, 1, nullptr, stream) : launch_few<false>(j, FewCe{e}, 1, nullptr, stream);
}

}  // namespace rnnt
