// Passes over memory of the linear layer and the output layer's cross entropy: padding, the epilogue's gradient, column sums, the rows that take part,
// statistics and score gradients.  All of them are bound by the bytes they move.
#include <algorithm>

#include "layers_device.h"

namespace rnnt {

namespace {

inline unsigned blocks_of(long long n, long long per) { return (unsigned)((n + per - 1) / per); }
inline bool grid_fits(long long n) { return n <= 0x7fffffffLL; }

// Padded copies, one thread per eight values: the workgroups of job k are [end[k - 1], end[k]) of those a launch has for them.
struct PadLaunch {
    PadJobs jobs;
    unsigned end[3];
};
PadLaunch pad_launch(const PadJobs& j) {
    PadLaunch p{j, {}};
    unsigned n = 0;
    for (int k = 0; k < 3; ++k) {
        if (k < j.n) n += (unsigned)std::min<long long>((j.job[k].rows_to * (j.job[k].ld_to / 8) + 255) / 256, 8192);
        p.end[k] = n;
    }
    return p;
}
__device__ __forceinline__ void pad_workgroup(const PadLaunch& p, unsigned block) {
    const int k = block >= p.end[1] ? 2 : block >= p.end[0] ? 1 : 0;
    const PadJob& j = p.jobs.job[k];
    const unsigned first = k == 2 ? p.end[1] : k == 1 ? p.end[0] : 0, wgs = p.end[k] - first;
    const long long groups = j.ld_to / 8, total = j.rows_to * groups;
    for (long long i = (long long)(block - first) * 256 + threadIdx.x; i < total; i += (long long)wgs * 256) {
        const long long r = i / groups, c = (i - r * groups) * 8;
        const long long left = j.r0 + r < j.rows ? j.cols - c : 0;
        const int live = left < 0 ? 0 : left < 8 ? (int)left : 8;
        const size_t from = (size_t)(j.r0 + r) * j.cols + c, to = (size_t)i * 8;
        if (j.kind == PAD_16) {
            *reinterpret_cast<bf16x8*>((bf16_t*)j.dst + to) = take8((const bf16_t*)j.src + (live ? from : 0), live);
        } else {
            float v[8];
            load8((const float*)j.src + (live ? from : 0), live, v);
            if (j.kind == PAD_PARTS) put_parts8((bf16_t*)j.dst + to, j.rows_to * j.ld_to, v);
            else store8((float*)j.dst + to, 8, v);
        }
    }
}
__global__ __launch_bounds__(256) void k_layer_pads(PadLaunch p) { pad_workgroup(p, blockIdx.x); }
__global__ __launch_bounds__(64) void k_layer_rng(const unsigned long long* __restrict__ state, unsigned long long* __restrict__ used) {
    if (threadIdx.x < 2) used[threadIdx.x] = state[threadIdx.x];
}

// The sums of 32 column granules over the eight thread rows of a workgroup -> part[n]
__device__ __forceinline__ void fold_columns(float (&sum)[8], float (*red)[256], float* __restrict__ part, int n, int N, int tid) {
    const int row = tid >> 5, g = tid & 31;
    *reinterpret_cast<f32x4*>(&red[row][g * 8]) = f32x4{sum[0], sum[1], sum[2], sum[3]};
    *reinterpret_cast<f32x4*>(&red[row][g * 8 + 4]) = f32x4{sum[4], sum[5], sum[6], sum[7]};
    __syncthreads();
    float t = 0.0f;
#pragma unroll
    for (int r = 0; r < 8; ++r) t += red[r][tid];
    if (n + tid < N) part[n + tid] = t;
}

// dz = dy act'(z) mask: a workgroup takes R rows x 256 columns, 8 thread rows x 32 granules of 8 columns.  The workgroups from dz_wgs on make the products'
// padded copies (a launch less: 1531 x 443 x 777, 4 us of 47).  Bound by bytes, with gelu' by its arithmetic too: 16000 x 4096, gelu, 93 us (4.2 TB/s);
// 8000 x 2048, silu, 18.6 us.
template <typename T, typename S>
__global__ __launch_bounds__(256) void k_layer_dz(DzArgs a, int R, int dz_wgs, PadLaunch pads) {
    constexpr bool FAST = sizeof(T) == 2;
    __shared__ __align__(16) float red[8][256];
    if ((int)blockIdx.x >= dz_wgs) return pad_workgroup(pads, blockIdx.x - dz_wgs);
    const int nb = (int)((a.ld + 255) / 256), rb = blockIdx.x / nb;
    const int tid = threadIdx.x, n0 = (blockIdx.x - rb * nb) * 256, n = n0 + (tid & 31) * 8;
    const long long r0 = (long long)rb * R;
    const int live = a.N - n < 0 ? 0 : a.N - n < 8 ? a.N - n : 8;
    float sum[8] = {};
#pragma unroll 2
    for (int i = 0; i < R / 8; ++i) {
        const long long m = r0 + i * 8 + (tid >> 5);
        if (m >= a.rows_to || n >= a.ld) break;
        float v[8] = {};
        if (m < a.M && live > 0) {
            const size_t at = (size_t)m * a.N + n;
            load8((const T*)a.dy + at, live, v);
            if (a.saved != nullptr) {
                float z[8];
                load8((const S*)a.saved + at, live, z);
                act_grad8<FAST>(a.act, z, v);
                // (a dropped entry, see saved8; one that was -infinity by itself has act' = 0)
                if (a.drop.cut != 0)
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] = z[j] == RNNT_NEG_INF ? 0.0f : v[j];
            } else if (a.drop.cut != 0) {
                bool keep[8];
                keep8(a.drop, m, n, keep);
                drop8(a.drop, keep, v);
            }
            if (live < 8)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = j < live ? v[j] : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] += v[j];
        if (a.dz != nullptr) {
            bf16_t* o = (bf16_t*)a.dz + (size_t)m * a.ld + n;     // (ld is a multiple of 64)
            if constexpr (sizeof(T) == 2) put_rounded8(o, a.rest, v);
            else put_parts8(o, a.rows_to * a.ld, v);
        }
    }
    if (a.part != nullptr && r0 < a.M) fold_columns(sum, red, a.part + (size_t)rb * a.ld, n0, a.N, tid);
}

// ---- cross entropy --------------------------------------------------------------------------------------------------
// The unit of the score gradients: the mantissa of the largest weight.  The label's gradient is w (p - 1), by far the largest of a row, and its rounding to bf16
// is off by up to 2^-8 where that lies just above a power of two, by the same for all rows where all have one weight and little p: a gradient's error was
// 0.0029 of it with weights of 1.01 / 1024.  Relative to the unit it is p - 1, which has 2^-9 at most.
__device__ __forceinline__ float unit_of(float largest) {
    return largest > 0.0f && largest < -RNNT_NEG_INF ? __uint_as_float((__float_as_uint(largest) & 0x007fffffu) | 0x3f800000u) : 1.0f;
}
// A workgroup numbers the real rows of its SCAN_ROWS behind those of the workgroups before it, which k_ce_count has counted (with their largest weight).
constexpr int SCAN_THREADS = 1024, SCAN_PER = CE_SCAN_ROWS / SCAN_THREADS;
__global__ __launch_bounds__(SCAN_THREADS) void k_ce_count(const int* __restrict__ labels, const float* __restrict__ weight, long long R, int ignore,
                                                           int2* __restrict__ counts) {
    __shared__ int wave_sum[SCAN_THREADS / 64];
    __shared__ float wave_most[SCAN_THREADS / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const long long first = (long long)blockIdx.x * CE_SCAN_ROWS;
    int n = 0;
    float most = 0.0f;
#pragma unroll
    for (int k = 0; k < SCAN_PER; ++k) {
        const long long i = first + k * SCAN_THREADS + tid;
        if (i >= R || labels[i] == ignore) continue;
        ++n;
        most = fmaxf(most, weight != nullptr ? fabsf(weight[i]) : 1.0f);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o, 64);
    most = wave_max(most);
    if (lane == 0) {
        wave_sum[wave] = n;
        wave_most[wave] = most;
    }
    __syncthreads();
    if (tid == 0) {
        for (int w = 1; w < SCAN_THREADS / 64; ++w) {
            n += wave_sum[w];
            most = fmaxf(most, wave_most[w]);
        }
        counts[blockIdx.x] = make_int2(n, __float_as_int(most));
    }
}
__global__ __launch_bounds__(SCAN_THREADS) void k_ce_rows(const int* __restrict__ labels, const float* __restrict__ weight, long long R, int ignore,
                                                          long long cap, const int2* __restrict__ counts, int* __restrict__ place, CeRows r) {
    __shared__ int wave_sum[SCAN_THREADS / 64], wave_before[SCAN_THREADS / 64];
    __shared__ float wave_most[SCAN_THREADS / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const long long first = (long long)blockIdx.x * CE_SCAN_ROWS;
    int before = 0;
    for (unsigned i = tid; i < blockIdx.x; i += SCAN_THREADS) before += counts[i].x;
    int y[SCAN_PER], mine = 0;
#pragma unroll
    for (int k = 0; k < SCAN_PER; ++k) {
        const long long i = first + tid * SCAN_PER + k;
        y[k] = i < R ? labels[i] : ignore;
        mine += y[k] != ignore;
    }
    int upto = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int t = __shfl_up(upto, o, 64);
        if (lane >= o) upto += t;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) before += __shfl_xor(before, o, 64);
    if (lane == 63) wave_sum[wave] = upto;
    if (lane == 0) wave_before[wave] = before;
    __syncthreads();
    int at = upto - mine, total = 0, prior = 0;
    for (int w = 0; w < SCAN_THREADS / 64; ++w) {
        prior += wave_before[w];
        total += wave_sum[w];
        if (w < wave) at += wave_sum[w];
    }
    at += prior;
    total += prior;
#pragma unroll
    for (int k = 0; k < SCAN_PER; ++k) {
        const long long i = first + tid * SCAN_PER + k;
        if (i >= R) break;
        const bool real = y[k] != ignore;
        place[i] = real ? at : -1;
        if (real) {
            r.index[at] = (int)i;
            r.label[at] = y[k];
            r.weight[at] = weight != nullptr ? weight[i] : 1.0f;
            ++at;
        }
    }
    if (blockIdx.x == gridDim.x - 1) {
        float most = 0.0f;
        for (unsigned i = tid; i < gridDim.x; i += SCAN_THREADS) most = fmaxf(most, __int_as_float(counts[i].y));
        most = wave_max(most);
        if (lane == 0) wave_most[wave] = most;
        __syncthreads();
        if (tid == 0) {
            for (int w = 0; w < SCAN_THREADS / 64; ++w) most = fmaxf(most, wave_most[w]);
            *r.count = total;
            *const_cast<float*>(ce_unit(r)) = unit_of(most);
        }
        // behind the last row: no label, no weight, up to the end of the arrays
        for (long long i = total + tid; i < cap; i += SCAN_THREADS) {
            r.index[i] = -1;
            r.label[i] = -1;
            r.weight[i] = 0.0f;
        }
    }
}

// A workgroup takes 16 rows of x, a wavefront four: their copies, or loss = 0 and dx = 0.  The FILL_WGS behind those fill what lies behind the last row; those
// behind them make W's padded copy.  12288 rows of 1024: 16 us (38 MB; the labels of all rows before are read by each workgroup).
// SCAN: a workgroup counts the real rows before its own itself (the labels come from the L2), which saves two launches; else k_ce_rows has left `place`.
constexpr int GATHER_ROWS = 16, FILL_WGS = 16;
typedef int i32x4_any __attribute__((ext_vector_type(4), aligned(4)));
// T: bf16, or float, whose rows go to xp as parts of cap rows.
template <typename T, bool SCAN>
__global__ __launch_bounds__(256) void k_ce_gather(const T* __restrict__ x, long long R, int D, const int* __restrict__ labels,
                                                   const float* __restrict__ weight, int ignore, long long cap, const int* __restrict__ place, CeRows r,
                                                   bf16_t* __restrict__ xp, long long ld, float* __restrict__ loss, T* __restrict__ dx, int row_wgs,
                                                   PadLaunch pads) {
    if ((int)blockIdx.x >= row_wgs + FILL_WGS) return pad_workgroup(pads, blockIdx.x - row_wgs - FILL_WGS);
    __shared__ int wave_count[4], at_row[GATHER_ROWS];
    __shared__ float wave_most[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const long long first = (long long)blockIdx.x * GATHER_ROWS;
    const bool fill = (int)blockIdx.x >= row_wgs;
    long long n = 0;                                              // real rows before this workgroup's, for the filling ones: all of them
    if constexpr (SCAN) {
        const long long upto = fill ? R : first;
        int c = 0;
        long long i = tid * 4;
#pragma unroll 4
        for (; i + 4 <= upto; i += 1024) {
            const i32x4_any y = *reinterpret_cast<const i32x4_any*>(labels + i);
            c += (y[0] != ignore) + (y[1] != ignore) + (y[2] != ignore) + (y[3] != ignore);
        }
        for (; i < upto; ++i) c += labels[i] != ignore;           // (one thread's last three at most)
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) c += __shfl_xor(c, o, 64);
        if (lane == 0) wave_count[wave] = c;
        __syncthreads();
        n = wave_count[0] + wave_count[1] + wave_count[2] + wave_count[3];
        if (!fill && tid < GATHER_ROWS) {
            const int y = first + tid < R ? labels[first + tid] : ignore;
            const bool real = y != ignore;
            const unsigned before = (unsigned)__ballot(real) & ((1u << tid) - 1u);
            const int at = (int)n + __popc(before);
            at_row[tid] = real ? at : -1;
            if (real) {
                r.index[at] = (int)(first + tid);
                r.label[at] = y;
                r.weight[at] = weight != nullptr ? weight[first + tid] : 1.0f;
            }
        }
        __syncthreads();
    } else if (fill) n = *r.count;
    if (!fill) {
#pragma unroll
        for (int k = 0; k < GATHER_ROWS / 4; ++k) {
            const long long row = first + wave * (GATHER_ROWS / 4) + k;
            if (row >= R) break;
            const int to = SCAN ? at_row[wave * (GATHER_ROWS / 4) + k] : place[row];
            const T* src = x + (size_t)row * D;
            if (to < 0) {
                if (lane == 0) loss[row] = 0.0f;
                if (dx != nullptr)
                    for (int c = lane; c < D; c += 64) dx[(size_t)row * D + c] = (T)0.0f;
                continue;
            }
            bf16_t* dst = xp + (size_t)to * ld;
            for (int c = lane * 8; c < ld; c += 512) {
                const int live = D - c < 0 ? 0 : D - c;
                if constexpr (sizeof(T) == 2) *reinterpret_cast<bf16x8*>(dst + c) = take8(src + (live ? c : 0), live);
                else {
                    float v[8];
                    load8(src + (live ? c : 0), live, v);
                    put_parts8(dst + c, cap * ld, v);
                }
            }
        }
        return;
    }
    // zeros behind the last row up to the next multiple of 256
    constexpr int wgs = FILL_WGS;
    const int wg = blockIdx.x - row_wgs;
    const long long end = (n + 255) / 256 * 256;
    for (long long at = n + wg * 4 + wave; at < end; at += wgs * 4)
        for (int c = lane * 8; c < ld; c += 512)
#pragma unroll
            for (int q = 0; q < (sizeof(T) == 2 ? 1 : PARTS); ++q) *reinterpret_cast<bf16x8*>(xp + q * cap * ld + (size_t)at * ld + c) = bf16x8{0};
    if constexpr (SCAN) {
        if (wg == 0) {
            float most = weight != nullptr ? 0.0f : 1.0f;
            if (weight != nullptr) {
                long long i = tid * 4;
#pragma unroll 4
                for (; i + 4 <= R; i += 1024) {
                    const i32x4_any y = *reinterpret_cast<const i32x4_any*>(labels + i);
                    const f32x4_at4 w = *reinterpret_cast<const f32x4_at4*>(weight + i);
#pragma unroll
                    for (int j = 0; j < 4; ++j) most = y[j] != ignore ? fmaxf(most, fabsf(w[j])) : most;
                }
                for (; i < R; ++i) most = labels[i] != ignore ? fmaxf(most, fabsf(weight[i])) : most;
            }
            most = wave_max(most);
            if (lane == 0) wave_most[wave] = most;
            __syncthreads();
            if (tid == 0) {
                *r.count = (int)n;
                *const_cast<float*>(ce_unit(r)) = unit_of(fmaxf(fmaxf(wave_most[0], wave_most[1]), fmaxf(wave_most[2], wave_most[3])));
            }
        }
        for (long long i = n + wg * 256 + tid; i < cap; i += wgs * 256) {
            r.index[i] = -1;
            r.label[i] = -1;
            r.weight[i] = 0.0f;
        }
    }
}

// Row i of a chunk: lse = M + ln(S / 2^15) out of the parts' statistics, loss = lse - score of the label (at < 0: not written); its scale.  The label's gradient
// w (p - 1) = w expm1(-loss): as good as the loss, about w 2^-20, where the kept exponential's p would leave it w 2^-12.
__device__ __forceinline__ float4 ce_finish_row(const CeChunk& c, long long i, int at, float M, float S) {
    const float m = M == RNNT_NEG_INF ? 0.0f : M;
    const int y = c.r.label[c.row0 + i];
    // (no entry of the vocabulary is possible, or the label is none of them: +inf)
    const bool none = S == 0.0f || (unsigned)y >= (unsigned)c.V;
    const float loss = none ? -RNNT_NEG_INF : (m - c.label_score[i]) + logf(S * 0x1p-15f);
    if (at >= 0) c.loss[at] = loss;
    const float w = c.identity ? 0.0f : c.r.weight[c.row0 + i] / *ce_unit(c.r);
    return make_float4(m, S == 0.0f ? 0.0f : w / S, w * expm1f(-loss), 0.0f);
}

// One wavefront per row (9288 rows, 128 parts: 11 us, as many bytes as a launch is long)
__global__ __launch_bounds__(256) void k_ce_finish(CeChunk c) {
    const long long i = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (i >= c.rows) return;
    const int lane = threadIdx.x & 63;
    int at;
    if (c.identity) {
        at = (int)i;
        if (c.r.label[i] == c.ignore) {
            if (lane == 0) c.loss[at] = 0.0f;
            return;
        }
    } else {
        at = c.r.index[c.row0 + i];
        if (at < 0) return;
    }
    const float2* st = c.stats + (size_t)i * c.tiles_n;
    float m = RNNT_NEG_INF;
    for (int t = lane; t < c.tiles_n; t += 64) m = fmaxf(m, st[t].x);
    const float M = wave_max(m), z = M == RNNT_NEG_INF ? 0.0f : M;
    float s = 0.0f;
    for (int t = lane; t < c.tiles_n; t += 64) s += st[t].y * __builtin_amdgcn_exp2f((st[t].x - z) * LOG2E_F);
    const float S = wave_sum(s);
    if (lane == 0) {
        const float4 f = ce_finish_row(c, i, at, M, S);
        if (c.scale != nullptr) c.scale[i] = f;
    }
}

// The kept exponentials times weight / sum and what brings their tile's maximum to the row's, the label's entry in place of its own; 2 + 2 bytes an entry: 9288 x
// 32768 240 us, 5.1 TB/s.  A workgroup takes R rows x 256 columns.  FINISH: it also forms its rows' sums, 256 / R threads for each (those of the first columns write the losses).
template <bool FINISH>
__global__ __launch_bounds__(256) void k_ce_grad(CeChunk c, void* __restrict__ kept, long long pitch, long long rest, float* __restrict__ part, int R) {
    __shared__ __align__(16) float red[8][256];
    __shared__ float4 scale[128];
    const int nb = (c.V + 255) / 256, rb = blockIdx.x / nb;
    const int tid = threadIdx.x, n0 = (blockIdx.x - rb * nb) * 256, n = n0 + (tid & 31) * 8;
    const long long r0 = (long long)rb * R;
    const CeRows& r = c.r;
    const long long row0 = c.row0;
    // rows up to the next multiple of 64 are read by the weight gradient's product: zeros there
    const long long real_rows = (long long)*r.count - row0, live = (real_rows + 63) / 64 * 64;
    if (r0 >= live || real_rows <= 0) return;
    if constexpr (FINISH) {
        const int per = 256 / R, in = tid / per, sub = tid & (per - 1);           // (R: a power of two from 16 to 128)
        const bool real = r0 + in < real_rows;
        const float2* st = c.stats + (size_t)(real ? r0 + in : 0) * c.tiles_n;
        // FINISH_LOADS of them at most, kept for the second pass
        float2 s[FINISH_LOADS];
        float M = RNNT_NEG_INF, S = 0.0f;
#pragma unroll
        for (int k = 0; k < FINISH_LOADS; ++k) s[k] = sub + k * per < c.tiles_n ? st[sub + k * per] : make_float2(RNNT_NEG_INF, 0.0f);
#pragma unroll
        for (int k = 0; k < FINISH_LOADS; ++k) M = fmaxf(M, s[k].x);
        for (int o = per >> 1; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor(M, o, 64));
        const float z = M == RNNT_NEG_INF ? 0.0f : M;
#pragma unroll
        for (int k = 0; k < FINISH_LOADS; ++k) S += s[k].y * __builtin_amdgcn_exp2f((s[k].x - z) * LOG2E_F);
        for (int o = per >> 1; o > 0; o >>= 1) S += __shfl_xor(S, o, 64);
        if (sub == 0)
            scale[in] = real ? ce_finish_row(c, r0 + in, n0 == 0 ? r.index[row0 + r0 + in] : -1, M, S) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    } else if (tid < R) scale[tid] = r0 + tid < real_rows ? c.scale[r0 + tid] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    __syncthreads();
    float sum[8] = {};
    const int t = n >> c.tile_log2;
    if (t < c.tiles_n)
#pragma unroll 4
        for (int i = 0; i < R / 8; ++i) {
            const int in = i * 8 + (tid >> 5);
            const long long m = r0 + in;
            if (m >= live) break;
            f16x8* at = reinterpret_cast<f16x8*>((_Float16*)kept + (size_t)m * pitch + n);
            float v[8] = {};
            if (m < real_rows) {
                const f16x8 h = *at;
                const float4 f = scale[in];
                // (a row without a possible entry has f.y = 0 and parts of -inf; its exponentials are zeros)
                const float k = f.y * __builtin_amdgcn_exp2f((c.stats[(size_t)m * c.tiles_n + t].x - f.x) * LOG2E_F);
                const int label = r.label[row0 + m], y = label < c.V ? label - n : -1;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    v[j] = y == j ? f.z : (float)h[j] * k;
                    sum[j] += v[j];
                }
            }
            put_rounded8(reinterpret_cast<bf16_t*>(at), rest, v);
        }
    if (part != nullptr) fold_columns(sum, red, part + (size_t)rb * pitch, n0, c.V, tid);
}

// fp32: a workgroup per row of scores: maximum, sum of the exponentials, then the gradient as parts (the row stays in the caches).  1748 x 4096: 20 us, 4.3 TB/s
// of 4 bytes read and 8 written an entry.
__global__ __launch_bounds__(256) void k_ce_rows_f32(CeRows r, long long row0, const float* __restrict__ scores, long long ld, int V,
                                                     float* __restrict__ loss, bf16_t* __restrict__ grad, long long part) {
    __shared__ float2 red[4];
    const long long i = blockIdx.x, count = (long long)*r.count - row0;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    bf16_t* g = grad + (size_t)i * ld;
    if (i >= count) {
        if (grad != nullptr && i < (count + 63) / 64 * 64)
            for (int v = tid * 8; v < ld; v += 2048)
#pragma unroll
                for (int q = 0; q < PARTS; ++q) *reinterpret_cast<bf16x8*>(g + q * part + v) = bf16x8{0};
        return;
    }
    const float* h = scores + (size_t)i * ld;
    const int at = r.index[row0 + i], y = r.label[row0 + i];
    const bool known = (unsigned)y < (unsigned)V;
    const float hy = known ? h[y] : 0.0f;
    auto each = [&](auto&& f) {                                    // (ld, and with it every row, is a multiple of 64 floats)
#pragma unroll 2
        for (int v = tid * 8; v < V; v += 2048) {
            float x[8];
            load8(h + v, 8, x);
            if (v + 8 > V)
#pragma unroll
                for (int k = 0; k < 8; ++k) x[k] = v + k < V ? x[k] : RNNT_NEG_INF;
            f(v, x);
        }
    };
    float m = RNNT_NEG_INF, s = 0.0f;
    each([&](int, const float (&x)[8]) {
#pragma unroll
        for (int k = 0; k < 8; ++k) m = fmaxf(m, x[k]);
    });
    m = wave_max(m);
    if (lane == 0) red[wave].x = m;
    __syncthreads();
    const float M = fmaxf(fmaxf(red[0].x, red[1].x), fmaxf(red[2].x, red[3].x)), c = M == RNNT_NEG_INF ? 0.0f : M;
    each([&](int, const float (&x)[8]) {
#pragma unroll
        for (int k = 0; k < 8; ++k) s += expf(x[k] - c);
    });
    s = wave_sum(s);
    if (lane == 0) red[wave].y = s;
    __syncthreads();
    const float S = (red[0].y + red[1].y) + (red[2].y + red[3].y);
    const float row_loss = S == 0.0f || !known ? -RNNT_NEG_INF : (c - hy) + logf(S);
    if (tid == 0) loss[at] = row_loss;
    if (grad == nullptr) return;
    const float w = r.weight[row0 + i], f = S == 0.0f ? 0.0f : w / S, of_label = w * expm1f(-row_loss);      // (w (p - 1), see ce_finish_row)
    each([&](int v, float (&x)[8]) {
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = v + k == y ? of_label : S == 0.0f ? 0.0f : expf(x[k] - c) * f;
        put_parts8(g + v, part, x);
    });
    for (int v = (V + 7) / 8 * 8 + tid * 8; v < ld; v += 2048)
#pragma unroll
        for (int q = 0; q < PARTS; ++q) *reinterpret_cast<bf16x8*>(g + q * part + v) = bf16x8{0};
}

__global__ __launch_bounds__(256) void k_layer_col_sums_f32(const bf16_t* __restrict__ x, long long rows, long long ld, int N, const int* __restrict__ count,
                                                            long long row0, float* __restrict__ part, int R) {
    __shared__ __align__(16) float red[8][256];
    const int nb = (N + 255) / 256, rb = blockIdx.x / nb;
    const int tid = threadIdx.x, n0 = (blockIdx.x - rb * nb) * 256, n = n0 + (tid & 31) * 8;
    const long long r0 = (long long)rb * R, live = (long long)*count - row0;
    if (r0 >= live) return;
    float sum[8] = {};
    if (n < ld)
#pragma unroll 4
        for (int i = 0; i < R / 8; ++i) {
            const long long m = r0 + i * 8 + (tid >> 5);
            if (m >= live) break;
            const bf16_t* p = x + (size_t)m * ld + n;
            const bf16x8 h = *reinterpret_cast<const bf16x8*>(p), q = *reinterpret_cast<const bf16x8*>(p + 2 * rows * ld),
                         l = *reinterpret_cast<const bf16x8*>(p + 3 * rows * ld);
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] += (float)h[j] + ((float)q[j] + (float)l[j]);
        }
    fold_columns(sum, red, part + (size_t)rb * ld, n0, N, tid);
}

// One workgroup: a fixed order; partial sums in fp64 (a sum of many losses of one size)
__global__ __launch_bounds__(1024) void k_ce_total(const float* __restrict__ loss, const float* __restrict__ weight, long long R, float* __restrict__ total) {
    __shared__ double part[16];
    double s = 0.0;
    // (both loads whatever the weight is: behind a branch they would follow each other)
    long long i = threadIdx.x * 4;
#pragma unroll 4
    for (; i + 4 <= R; i += 4096) {
        const f32x4_at4 l = *reinterpret_cast<const f32x4_at4*>(loss + i);
        f32x4 w = f32x4{1.0f, 1.0f, 1.0f, 1.0f};
        if (weight != nullptr) w = *reinterpret_cast<const f32x4_at4*>(weight + i);
#pragma unroll
        for (int j = 0; j < 4; ++j) s += w[j] != 0.0f ? (double)w[j] * (double)l[j] : 0.0;
    }
    for (; i < R; ++i) {                                           // (one thread's last three at most)
        const float w = weight != nullptr ? weight[i] : 1.0f;
        s += w != 0.0f ? (double)w * (double)loss[i] : 0.0;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        double t = 0.0;
        for (int w = 0; w < 16; ++w) t += part[w];
        *total = (float)t;
    }
}

// (bf16 gradients are rounded once more, where the factor is no power of two: the alternative is computing them again)
struct ScaleArgs {
    void* p[3];
    long long n[3];
    bool bf16[3];
};
__global__ __launch_bounds__(256) void k_layer_scale(const float* __restrict__ factor, ScaleArgs a) {
    const float f = *factor;
    if (f == 1.0f) return;
#pragma unroll
    for (int k = 0; k < 3; ++k)
        for (long long i = ((long long)blockIdx.x * 256 + threadIdx.x) * 8; i < a.n[k]; i += (long long)gridDim.x * 2048) {
            const int live = a.n[k] - i < 8 ? (int)(a.n[k] - i) : 8;
            float v[8];
            if (a.bf16[k]) load8((const bf16_t*)a.p[k] + i, live, v);
            else load8((const float*)a.p[k] + i, live, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= f;
            if (a.bf16[k]) store8((bf16_t*)a.p[k] + i, live, v);
            else store8((float*)a.p[k] + i, live, v);
        }
}

}  // namespace

hipError_t launch_ce_total(const float* loss, const float* weight, long long R, float* total, hipStream_t stream) {
    k_ce_total<<<dim3(1), dim3(1024), 0, stream>>>(loss, weight, R, total);
    return hipGetLastError();
}
hipError_t launch_scale(const float* factor, void* const (&p)[3], const long long (&n)[3], const bool (&bf16)[3], hipStream_t stream) {
    ScaleArgs a;
    long long most = 0;
    for (int k = 0; k < 3; ++k) {
        a.p[k] = p[k];
        a.n[k] = n[k];
        a.bf16[k] = bf16[k];
        most = std::max(most, n[k]);
    }
    if (most == 0) return hipSuccess;
    k_layer_scale<<<dim3((unsigned)std::min<long long>(2048, (most + 2047) / 2048)), dim3(256), 0, stream>>>(factor, a);
    return hipGetLastError();
}

hipError_t launch_pads(const PadJobs& j, hipStream_t stream) {
    const PadLaunch p = pad_launch(j);
    if (p.end[2] == 0) return hipSuccess;
    k_layer_pads<<<dim3(p.end[2]), dim3(256), 0, stream>>>(p);
    return hipGetLastError();
}

hipError_t launch_pass_rng(const unsigned long long* state, unsigned long long* used, hipStream_t stream) {
    k_layer_rng<<<dim3(1), dim3(64), 0, stream>>>(state, used);
    return hipGetLastError();
}

hipError_t launch_dz(bool bf16, const DzArgs& a, const PadJobs& pads, hipStream_t stream) {
    const int R = sum_rows(a.M, a.N);
    const PadLaunch p = pad_launch(pads);
    const long long n = (std::max(a.M, a.rows_to) + R - 1) / R * ((a.ld + 255) / 256);
    if (!grid_fits(n + p.end[2])) return hipErrorInvalidValue;
    const dim3 grid((unsigned)n + p.end[2]);
    if (bf16) k_layer_dz<bf16_t, _Float16><<<grid, dim3(256), 0, stream>>>(a, R, (int)n, p);
    else k_layer_dz<float, float><<<grid, dim3(256), 0, stream>>>(a, R, (int)n, p);
    return hipGetLastError();
}

namespace {
template <typename T>
hipError_t gather(const void* x, long long R, int D, const int* labels, const float* weight, int ignore, long long cap, int* place, const CeRows& r, void* xp,
                  long long ld, float* loss, void* dx, const PadJobs& pads, hipStream_t stream) {
    const unsigned row_wgs = blocks_of(R, GATHER_ROWS);
    const PadLaunch p = pad_launch(pads);
    const dim3 grid(row_wgs + FILL_WGS + p.end[2]);
    if (R <= GATHER_SCAN) {
        k_ce_gather<T, true><<<grid, dim3(256), 0, stream>>>((const T*)x, R, D, labels, weight, ignore, cap, nullptr, r, (bf16_t*)xp, ld, loss, (T*)dx,
                                                             (int)row_wgs, p);
    } else {
        int2* counts = reinterpret_cast<int2*>(place + cap);
        k_ce_count<<<dim3(blocks_of(R, CE_SCAN_ROWS)), dim3(SCAN_THREADS), 0, stream>>>(labels, weight, R, ignore, counts);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        k_ce_rows<<<dim3(blocks_of(R, CE_SCAN_ROWS)), dim3(SCAN_THREADS), 0, stream>>>(labels, weight, R, ignore, cap, counts, place, r);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
        k_ce_gather<T, false><<<grid, dim3(256), 0, stream>>>((const T*)x, R, D, labels, weight, ignore, cap, place, r, (bf16_t*)xp, ld, loss, (T*)dx,
                                                              (int)row_wgs, p);
    }
    return hipGetLastError();
}
}  // namespace
hipError_t launch_ce_gather(const void* x, bool f32, long long R, int D, const int* labels, const float* weight, int ignore, long long cap, int* place,
                            const CeRows& r, void* xp, long long ld, float* loss, void* dx, const PadJobs& pads, hipStream_t stream) {
    return f32 ? gather<float>(x, R, D, labels, weight, ignore, cap, place, r, xp, ld, loss, dx, pads, stream)
               : gather<bf16_t>(x, R, D, labels, weight, ignore, cap, place, r, xp, ld, loss, dx, pads, stream);
}
hipError_t launch_ce_finish(const CeChunk& c, hipStream_t stream) {
    k_ce_finish<<<dim3(blocks_of(c.rows, 4)), dim3(256), 0, stream>>>(c);
    return hipGetLastError();
}
hipError_t launch_ce_grad(const CeChunk& c, void* kept, long long pitch, long long rest, float* part, hipStream_t stream) {
    const int R = sum_rows(c.rows, c.V);
    const long long n = (long long)blocks_of(c.V, 256) * sum_blocks(c.rows, c.V);
    if (!grid_fits(n)) return hipErrorInvalidValue;
    if (ce_grad_finishes(c.rows, c.V, c.tiles_n)) k_ce_grad<true><<<dim3((unsigned)n), dim3(256), 0, stream>>>(c, kept, pitch, rest, part, R);
    else k_ce_grad<false><<<dim3((unsigned)n), dim3(256), 0, stream>>>(c, kept, pitch, rest, part, R);
    return hipGetLastError();
}
hipError_t launch_ce_rows_f32(const CeRows& r, long long row0, long long rows, const float* scores, long long ld, int V, float* loss, void* grad,
                              hipStream_t stream) {
    k_ce_rows_f32<<<dim3((unsigned)rows), dim3(256), 0, stream>>>(r, row0, scores, ld, V, loss, (bf16_t*)grad, rows * ld);
    return hipGetLastError();
}
hipError_t launch_col_sums_f32(const void* x, long long rows, long long ld, int N, const int* count, long long row0, float* part, hipStream_t stream) {
    const int R = sum_rows(rows, N);
    const long long n = (long long)blocks_of(N, 256) * sum_blocks(rows, N);
    if (!grid_fits(n)) return hipErrorInvalidValue;
    k_layer_col_sums_f32<<<dim3((unsigned)n), dim3(256), 0, stream>>>((const bf16_t*)x, rows, ld, N, count, row0, part, R);
    return hipGetLastError();
}

}  // namespace rnnt
