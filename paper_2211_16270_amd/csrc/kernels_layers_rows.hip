// Passes over memory of the linear layer and the output layer's cross entropy: padding, the epilogue's gradient, column sums, the rows that take part,
// statistics and score gradients.  All of them are bound by the bytes they move.
#include <algorithm>

#include "layers_device.h"

namespace rnnt {

namespace {

inline unsigned blocks_of(long long n, long long per) { return (unsigned)((n + per - 1) / per); }
inline bool grid_fits(long long n) { return n <= 0x7fffffffLL; }

template <typename T>
__global__ __launch_bounds__(256) void k_layer_pad(const T* __restrict__ src, long long rows, long long cols, long long r0, T* __restrict__ dst,
                                                   long long ld_to, long long total) {
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < total; i += (long long)gridDim.x * 256) {
        const long long r = i / ld_to, c = i - r * ld_to;
        dst[i] = r0 + r < rows && c < cols ? src[(r0 + r) * cols + c] : (T)0;
    }
}

// Eight consecutive values of a row, as floats
template <typename T>
__device__ __forceinline__ void load8(const T* p, int live, bool vec, float (&v)[8]) {
    if (vec) {
        if constexpr (sizeof(T) == 2) {
            typedef T t8 __attribute__((ext_vector_type(8)));
            const t8 x = *reinterpret_cast<const t8*>(p);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = (float)x[j];
        } else {
            const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[j] = a[j];
                v[4 + j] = b[j];
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = j < live ? (float)p[j] : 0.0f;
    }
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

// dz = dy act'(z) mask / (1 - p): a workgroup takes 128 rows x 256 columns, 8 thread rows x 32 granules of 8 columns.
template <typename T, typename S>
__global__ __launch_bounds__(256) void k_layer_dz(DzArgs a) {
    constexpr bool FAST = sizeof(T) == 2;
    __shared__ __align__(16) float red[8][256];
    const int nb = (int)((a.ld + 255) / 256), rb = blockIdx.x / nb;
    const int tid = threadIdx.x, n0 = (blockIdx.x - rb * nb) * 256, n = n0 + (tid & 31) * 8;
    const long long r0 = (long long)rb * SUM_ROWS;
    const int live = a.N - n < 0 ? 0 : a.N - n < 8 ? a.N - n : 8;
    float sum[8] = {};
#pragma unroll 2
    for (int i = 0; i < SUM_ROWS / 8; ++i) {
        const long long m = r0 + i * 8 + (tid >> 5);
        if (m >= a.rows_to || n >= a.ld) break;
        float v[8] = {};
        if (m < a.M && live > 0) {
            const size_t at = (size_t)m * a.N + n;
            load8((const T*)a.dy + at, live, a.vec && live == 8, v);
            if (a.saved != nullptr) {
                float z[8];
                load8((const S*)a.saved + at, live, a.vec && live == 8, z);
                act_grad8<FAST>(a.act, z, v);
            }
            drop8(a.drop, m, n, v);
            if (live < 8)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = j < live ? v[j] : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] += v[j];
        if (a.dz != nullptr) {
            T* o = (T*)a.dz + (size_t)m * a.ld + n;               // (ld is a multiple of 64, fp32: of 4)
            if constexpr (sizeof(T) == 2) {
                bf16x8 x;
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = (bf16_t)v[j];
                *reinterpret_cast<bf16x8*>(o) = x;
            } else {
                *reinterpret_cast<f32x4*>(o) = f32x4{v[0], v[1], v[2], v[3]};
                if (n + 4 < a.ld) *reinterpret_cast<f32x4*>(o + 4) = f32x4{v[4], v[5], v[6], v[7]};
            }
        }
    }
    if (a.part != nullptr && r0 < a.M) fold_columns(sum, red, a.part + (size_t)rb * a.ld, n0, a.N, tid);
}

// 32 columns x 8 thread rows per workgroup; the partial sums are added in a fixed order
template <typename O>
__global__ __launch_bounds__(256) void k_layer_sum_parts(const float* __restrict__ part, int blocks, long long ld, int N, const int* __restrict__ count,
                                                         long long row0, const float* __restrict__ prev, O* __restrict__ out) {
    __shared__ float red[8][32];
    const int c = threadIdx.x & 31, row = threadIdx.x >> 5, n = blockIdx.x * 32 + c;
    if (count != nullptr) {
        long long r = (long long)*count - row0;
        r = r < 0 ? 0 : (r + SUM_ROWS - 1) / SUM_ROWS;
        blocks = r < blocks ? (int)r : blocks;
    }
    float s = 0.0f;
    if (n < N)
        for (int b = row; b < blocks; b += 8) s += part[(size_t)b * ld + n];
    red[row][c] = s;
    __syncthreads();
    if (row == 0 && n < N) {
        float t = prev != nullptr ? prev[n] : 0.0f;
#pragma unroll
        for (int r = 0; r < 8; ++r) t += red[r][c];
        out[n] = (O)t;
    }
}

// z (pitch ld, may be saved or y) + bias -> saved, y; one thread per eight columns
__global__ __launch_bounds__(256) void k_linear_rows_f32(const float* z, long long ld, const float* __restrict__ bias, const float* __restrict__ residual,
                                                         float* y, float* saved, long long M, int N, int act, Dropout drop, long long groups,
                                                         long long total) {
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i >= total) return;
    const long long m = i / groups;
    const int n = (int)(i - m * groups) * 8, live = N - n < 8 ? N - n : 8;
    const size_t at = (size_t)m * N + n;
    const bool vec = live == 8 && N % 4 == 0;
    float v[8], b[8];
    load8(z + (size_t)m * ld + n, live, vec, v);
    load_bias8(bias, n, N, b);
    auto store8 = [&](float* to) {
        if (vec) {
            *reinterpret_cast<f32x4*>(to + at) = f32x4{v[0], v[1], v[2], v[3]};
            *reinterpret_cast<f32x4*>(to + at + 4) = f32x4{v[4], v[5], v[6], v[7]};
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < live) to[at + j] = v[j];
        }
    };
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += b[j];
    if (saved != nullptr) store8(saved);
    act8<false>(act, v);
    drop8(drop, m, n, v);
    if (residual != nullptr) {
        float r[8];
        load8(residual + at, live, vec, r);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += r[j];
    }
    store8(y);
}

__global__ __launch_bounds__(256) void k_layer_crop_f32(const float* __restrict__ src, long long ld, float* __restrict__ dst, int N, long long total,
                                                        bool add) {
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < total; i += (long long)gridDim.x * 256) {
        const long long r = i / N;
        const float v = src[r * ld + (i - r * N)];
        dst[i] = add ? dst[i] + v : v;
    }
}

// ---- cross entropy --------------------------------------------------------------------------------------------------
// Each workgroup counts the real rows before its own SCAN_ROWS (the labels come from the L2) and numbers its own.
constexpr int SCAN_THREADS = 1024, SCAN_PER = 4, SCAN_ROWS = SCAN_THREADS * SCAN_PER;
__global__ __launch_bounds__(SCAN_THREADS) void k_ce_rows(const int* __restrict__ labels, const float* __restrict__ weight, long long R, int ignore,
                                                          long long cap, CeRows r) {
    __shared__ int wave_sum[SCAN_THREADS / 64], wave_before[SCAN_THREADS / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const long long first = (long long)blockIdx.x * SCAN_ROWS;
    int before = 0;
    for (long long i = tid; i < first; i += SCAN_THREADS) before += labels[i] != ignore;
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
        r.place[i] = real ? at : -1;
        if (real) {
            r.index[at] = (int)i;
            r.label[at] = y[k];
            r.weight[at] = weight != nullptr ? weight[i] : 1.0f;
            ++at;
        }
    }
    if (blockIdx.x == gridDim.x - 1) {
        if (tid == 0) *r.count = total;
        // behind the last row: no label, no weight, up to the end of the arrays
        for (long long i = total + tid; i < cap; i += SCAN_THREADS) {
            r.index[i] = -1;
            r.label[i] = -1;
            r.weight[i] = 0.0f;
        }
    }
}

// One wavefront per row of x (its copy, or loss = 0 and dx = 0), then per row behind the last
template <typename T>
__global__ __launch_bounds__(256) void k_ce_gather(const T* __restrict__ x, long long R, int D, CeRows r, T* __restrict__ xp, long long ld,
                                                   long long fill_to, float* __restrict__ loss, T* __restrict__ dx, bool vec) {
    const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    constexpr int E = 16 / sizeof(T);
    typedef T piece __attribute__((ext_vector_type(E)));
    if (row < R) {
        const int to = r.place[row];
        const T* src = x + (size_t)row * D;
        if (to < 0) {
            if (lane == 0) loss[row] = 0.0f;
            if (dx != nullptr)
                for (int c = lane; c < D; c += 64) dx[(size_t)row * D + c] = (T)0;
            return;
        }
        T* dst = xp + (size_t)to * ld;
        if (vec) {
            for (int c = lane * E; c < D; c += 64 * E) *reinterpret_cast<piece*>(dst + c) = *reinterpret_cast<const piece*>(src + c);
            for (int c = D + lane; c < ld; c += 64) dst[c] = (T)0;
        } else {
            for (int c = lane; c < ld; c += 64) dst[c] = c < D ? src[c] : (T)0;
        }
        return;
    }
    // zeros behind the last row, up to fill_to (0: the next multiple of 256)
    const long long n = *r.count, end = fill_to != 0 ? fill_to : (n + 255) / 256 * 256, at = n + (row - R);
    if (at < end)
        for (int c = lane; c < ld; c += 64) xp[(size_t)at * ld + c] = (T)0;
}

// One wavefront per row: lse = M + ln(S / 2^15) out of the tiles' statistics, loss = lse - score of the label, and per tile the factor that makes
// weight * probability of a kept exponential.
__global__ __launch_bounds__(256) void k_ce_finish(CeRows r, long long row0, long long rows, const float* __restrict__ label_score,
                                                   float2* __restrict__ stats, int tiles_n, int V, float* __restrict__ loss, bool grads) {
    const long long i = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (i >= rows) return;
    const int lane = threadIdx.x & 63, at = r.index[row0 + i];
    float2* st = stats + (size_t)i * tiles_n;
    if (at < 0) return;
    float m = RNNT_NEG_INF;
    for (int t = lane; t < tiles_n; t += 64) m = fmaxf(m, st[t].x);
    const float M = wave_max(m), c = M == RNNT_NEG_INF ? 0.0f : M;
    float s = 0.0f;
    for (int t = lane; t < tiles_n; t += 64) s += st[t].y * __builtin_amdgcn_exp2f((st[t].x - c) * LOG2E_F);
    const float S = wave_sum(s);
    if (lane == 0) {
        const int y = r.label[row0 + i];
        // (no entry of the vocabulary is possible, or the label is none of them: +inf)
        const bool none = S == 0.0f || (unsigned)y >= (unsigned)V;
        loss[at] = none ? -RNNT_NEG_INF : (c - label_score[i]) + LN2_F * (__builtin_amdgcn_logf(S) - 15.0f);
    }
    if (!grads) return;
    const float w = S == 0.0f ? 0.0f : r.weight[row0 + i] / S;
    for (int t = lane; t < tiles_n; t += 64) st[t].x = S == 0.0f ? 0.0f : w * __builtin_amdgcn_exp2f((st[t].x - c) * LOG2E_F);
}

// A workgroup takes 128 rows x 256 columns
__global__ __launch_bounds__(256) void k_ce_grad(CeRows r, long long row0, void* __restrict__ kept, long long pitch, const float2* __restrict__ stats,
                                                 int tiles_n, int tile_log2, int V, float* __restrict__ part, long long part_ld) {
    __shared__ __align__(16) float red[8][256];
    const int nb = (V + 255) / 256, rb = blockIdx.x / nb;
    const int tid = threadIdx.x, n0 = (blockIdx.x - rb * nb) * 256, n = n0 + (tid & 31) * 8;
    const long long r0 = (long long)rb * SUM_ROWS;
    long long live = (long long)*r.count - row0;
    if (r0 >= live) return;
    // rows up to the next multiple of 64 are read by the weight gradient's product: zeros there (their exponentials are finite, their weight 0)
    live = (live + 63) / 64 * 64;
    float sum[8] = {};
    const int t = n >> tile_log2;
    if (t < tiles_n)
#pragma unroll 4
        for (int i = 0; i < SUM_ROWS / 8; ++i) {
            const long long m = r0 + i * 8 + (tid >> 5);
            if (m >= live) break;
            f16x8* at = reinterpret_cast<f16x8*>((_Float16*)kept + (size_t)m * pitch + n);
            const f16x8 h = *at;
            const float w = r.weight[row0 + m];
            const bool real = r.index[row0 + m] >= 0;
            const float f = real ? stats[(size_t)m * tiles_n + t].x : 0.0f;
            const int y = r.label[row0 + m] - n;
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[j] = real ? (float)h[j] * f : 0.0f;
                if (y == j) v[j] -= w;
                sum[j] += v[j];
            }
            bf16x8 o;
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = (bf16_t)v[j];
            *reinterpret_cast<bf16x8*>(at) = o;
        }
    if (part != nullptr) fold_columns(sum, red, part + (size_t)rb * part_ld, n0, V, tid);
}

// fp32: a workgroup per row of scores: maximum and sum of the exponentials in one pass, the gradient in a second one
__global__ __launch_bounds__(256) void k_ce_rows_f32(CeRows r, long long row0, float* __restrict__ scores, long long ld, int V,
                                                     const float* __restrict__ b, float* __restrict__ loss, bool grads) {
    __shared__ float2 part[4];
    const long long i = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, at = r.index[row0 + i];
    float* h = scores + (size_t)i * ld;
    f32x4* h4 = reinterpret_cast<f32x4*>(h);
    if (at < 0) {
        if (grads)
            for (int v = tid; v < ld / 4; v += 256) h4[v] = f32x4{0};
        return;
    }
    const int y = r.label[row0 + i];
    const bool known = (unsigned)y < (unsigned)V;
    auto score = [&](int v) { return b != nullptr ? h[v] + b[v] : h[v]; };
    const float hy = known ? score(y) : 0.0f;
    float m = RNNT_NEG_INF, s = 0.0f;
    for (int v = tid; v < V; v += 256) m = fmaxf(m, score(v));
    m = wave_max(m);
    if (lane == 0) part[wave].x = m;
    __syncthreads();
    const float M = fmaxf(fmaxf(part[0].x, part[1].x), fmaxf(part[2].x, part[3].x)), c = M == RNNT_NEG_INF ? 0.0f : M;
    for (int v = tid; v < V; v += 256) s += expf(score(v) - c);
    s = wave_sum(s);
    if (lane == 0) part[wave].y = s;
    __syncthreads();
    const float S = (part[0].y + part[1].y) + (part[2].y + part[3].y);
    if (tid == 0) loss[at] = S == 0.0f || !known ? -RNNT_NEG_INF : (c - hy) + logf(S);
    if (!grads) return;
    const float w = r.weight[row0 + i], f = S == 0.0f ? 0.0f : w / S;
    for (int v = tid; v < ld; v += 256) {
        float d = v < V && S != 0.0f ? expf(score(v) - c) * f : 0.0f;
        if (v == y && known) d -= w;
        h[v] = d;
    }
}

__global__ __launch_bounds__(256) void k_layer_col_sums_f32(const float* __restrict__ x, long long rows, long long ld, int N, float* __restrict__ part) {
    __shared__ __align__(16) float red[8][256];
    const int nb = (N + 255) / 256, rb = blockIdx.x / nb;
    const int tid = threadIdx.x, n0 = (blockIdx.x - rb * nb) * 256, n = n0 + (tid & 31) * 8;
    const int live = ld - n < 8 ? (int)(ld - n) : 8;
    const long long r0 = (long long)rb * SUM_ROWS;
    float sum[8] = {};
    if (n < ld)
#pragma unroll 4
        for (int i = 0; i < SUM_ROWS / 8; ++i) {
            const long long m = r0 + i * 8 + (tid >> 5);
            if (m >= rows) break;
            float v[8];
            load8(x + (size_t)m * ld + n, live, live == 8, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] += v[j];
        }
    fold_columns(sum, red, part + (size_t)rb * ld, n0, N, tid);
}

__global__ __launch_bounds__(256) void k_ce_scatter_f32(CeRows r, long long row0, long long rows, const float* __restrict__ src, long long ld, int D,
                                                        float* __restrict__ dx) {
    const long long i = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (i >= rows) return;
    const int at = r.index[row0 + i];
    if (at < 0) return;
    for (int c = threadIdx.x & 63; c < D; c += 64) dx[(size_t)at * D + c] = src[(size_t)i * ld + c];
}

}  // namespace

hipError_t launch_pad(const void* src, int size, long long rows, long long cols, long long r0, void* dst, long long rows_to, long long ld_to,
                      hipStream_t stream) {
    const long long total = rows_to * ld_to;
    if (total <= 0) return hipSuccess;
    const unsigned grid = (unsigned)std::min<long long>((total + 255) / 256, 16384);
    if (size == 2)
        k_layer_pad<unsigned short><<<dim3(grid), dim3(256), 0, stream>>>((const unsigned short*)src, rows, cols, r0, (unsigned short*)dst, ld_to, total);
    else k_layer_pad<unsigned><<<dim3(grid), dim3(256), 0, stream>>>((const unsigned*)src, rows, cols, r0, (unsigned*)dst, ld_to, total);
    return hipGetLastError();
}

hipError_t launch_dz(bool bf16, const DzArgs& a, hipStream_t stream) {
    const long long n = (std::max(a.M, a.rows_to) + SUM_ROWS - 1) / SUM_ROWS * ((a.ld + 255) / 256);
    if (!grid_fits(n)) return hipErrorInvalidValue;
    const dim3 grid((unsigned)n);
    if (bf16) k_layer_dz<bf16_t, _Float16><<<grid, dim3(256), 0, stream>>>(a);
    else k_layer_dz<float, float><<<grid, dim3(256), 0, stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_sum_parts(const float* part, int blocks, long long ld, int N, const int* count, long long row0, const float* prev, void* out,
                            bool bf16, hipStream_t stream) {
    if (N <= 0) return hipSuccess;
    const dim3 grid(blocks_of(N, 32));
    if (bf16) k_layer_sum_parts<bf16_t><<<grid, dim3(256), 0, stream>>>(part, blocks, ld, N, count, row0, prev, (bf16_t*)out);
    else k_layer_sum_parts<float><<<grid, dim3(256), 0, stream>>>(part, blocks, ld, N, count, row0, prev, (float*)out);
    return hipGetLastError();
}

hipError_t launch_linear_rows_f32(const float* z, long long ld, const float* bias, const float* residual, float* y, float* saved, long long M, int N,
                                  int act, const Dropout& drop, hipStream_t stream) {
    const long long groups = (N + 7) / 8, total = M * groups;
    if (total <= 0) return hipSuccess;
    if (!grid_fits((total + 255) / 256)) return hipErrorInvalidValue;
    k_linear_rows_f32<<<dim3(blocks_of(total, 256)), dim3(256), 0, stream>>>(z, ld, bias, residual, y, saved, M, N, act, drop, groups, total);
    return hipGetLastError();
}
hipError_t launch_crop_f32(const float* src, long long ld, float* dst, long long rows, int N, bool add, hipStream_t stream) {
    const long long total = rows * N;
    if (total <= 0) return hipSuccess;
    k_layer_crop_f32<<<dim3((unsigned)std::min<long long>((total + 255) / 256, 16384)), dim3(256), 0, stream>>>(src, ld, dst, N, total, add);
    return hipGetLastError();
}

hipError_t launch_ce_rows(const int* labels, const float* weight, long long R, int ignore, long long cap, const CeRows& r, hipStream_t stream) {
    k_ce_rows<<<dim3(blocks_of(R, SCAN_ROWS)), dim3(SCAN_THREADS), 0, stream>>>(labels, weight, R, ignore, cap, r);
    return hipGetLastError();
}
hipError_t launch_ce_gather(const void* x, int size, long long R, int D, const CeRows& r, void* xp, long long ld, long long fill_to, float* loss, void* dx,
                            hipStream_t stream) {
    const bool vec = ((size_t)D * size) % 16 == 0;
    const dim3 grid(blocks_of(R + std::max(256LL, fill_to), 4));
    if (size == 2)
        k_ce_gather<unsigned short><<<grid, dim3(256), 0, stream>>>((const unsigned short*)x, R, D, r, (unsigned short*)xp, ld, fill_to, loss,
                                                                    (unsigned short*)dx, vec);
    else k_ce_gather<unsigned><<<grid, dim3(256), 0, stream>>>((const unsigned*)x, R, D, r, (unsigned*)xp, ld, fill_to, loss, (unsigned*)dx, vec);
    return hipGetLastError();
}
hipError_t launch_ce_finish(const CeRows& r, long long row0, long long rows, const float* label_score, float2* stats, int tiles_n, int V, float* loss,
                            bool grads, hipStream_t stream) {
    k_ce_finish<<<dim3(blocks_of(rows, 4)), dim3(256), 0, stream>>>(r, row0, rows, label_score, stats, tiles_n, V, loss, grads);
    return hipGetLastError();
}
hipError_t launch_ce_grad(const CeRows& r, long long row0, long long rows, void* kept, long long pitch, const float2* stats, int tiles_n, int tile, int V,
                          float* part, hipStream_t stream) {
    const long long n = (long long)blocks_of(V, 256) * blocks_of(rows, SUM_ROWS);
    if (!grid_fits(n)) return hipErrorInvalidValue;
    const dim3 grid((unsigned)n);
    k_ce_grad<<<grid, dim3(256), 0, stream>>>(r, row0, kept, pitch, stats, tiles_n, tile == 256 ? 8 : 7, V, part, pitch);
    return hipGetLastError();
}
hipError_t launch_ce_rows_f32(const CeRows& r, long long row0, long long rows, float* scores, long long ld, int V, const float* b, float* loss,
                              bool grads, hipStream_t stream) {
    k_ce_rows_f32<<<dim3((unsigned)rows), dim3(256), 0, stream>>>(r, row0, scores, ld, V, b, loss, grads);
    return hipGetLastError();
}
hipError_t launch_col_sums_f32(const float* x, long long rows, long long ld, int N, float* part, hipStream_t stream) {
    const long long n = (long long)blocks_of(N, 256) * blocks_of(rows, SUM_ROWS);
    if (!grid_fits(n)) return hipErrorInvalidValue;
    const dim3 grid((unsigned)n);
    k_layer_col_sums_f32<<<grid, dim3(256), 0, stream>>>(x, rows, ld, N, part);
    return hipGetLastError();
}
hipError_t launch_scatter_f32(const CeRows& r, long long row0, long long rows, const float* src, long long ld, int D, float* dx, hipStream_t stream) {
    k_ce_scatter_f32<<<dim3(blocks_of(rows, 4)), dim3(256), 0, stream>>>(r, row0, rows, src, ld, D, dx);
    return hipGetLastError();
}

}  // namespace rnnt
