// Internal launch interface of the layers beside the transducer loss (linear layer with its epilogue, output-layer cross entropy) between
// layers.cpp and the kernels.  Every function enqueues on `stream` and returns the launch status; none synchronises.
#pragma once
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

namespace rnnt {

enum Activation { ACT_NONE = 0, ACT_RELU, ACT_SILU, ACT_GELU, ACT_TANH, ACT_COUNT };

// Dropout: entry (m, n) draws 16 bits u of Philox4x32-10 and is kept where u >= cut, times scale = 65536 / (65536 - cut).  cut = 0: no dropout.
struct Dropout {
    const unsigned long long* state;     // device, {seed, offset}
    unsigned cut;
    float scale;
};

// ---- bf16 matrix products ---------------------------------------------------------------------------------------------
struct GemmOperand {
    const void* p;
    long long ld;                        // elements
    const void* tail;                    // k-slow operands whose K is no multiple of 64: the last stage's 64 rows, zeros from K on; else null
    int tail_stage;
};
// C[m, n] = sum_k A(m, k) B(k, n); a k-slow operand's extent along the other index is a multiple of 8, a k-contiguous one's K a multiple of 64.
// limit: a count of rows that only the device knows, n = max(0, min(*count - row0, extent)): it bounds M (GEMM_ROWS_M) or K (GEMM_ROWS_K, the operands
// being zero from there to the next multiple of 64).
enum GemmLimit { GEMM_FIXED = 0, GEMM_ROWS_M, GEMM_ROWS_K };
struct GemmJob {
    GemmOperand A, B;
    long long M, N;                      // tiles cover them; operands may be read up to a_rows, b_rows along their other index
    long long a_rows, b_rows;
    int stages;                          // ceil(K / 64)
    int limit;
    const int* count;
    long long row0;
};
struct GemmPlan {
    int tile;                            // 256 or 128
    int splits;                          // of the sum over k; each takes per_split stages
    int per_split;
};
// The tile and the splits that take least time (see there); slots of all splits together at most slot_cap bytes.
GemmPlan plan_gemm(long long M, long long N, int stages, size_t slot_cap);
inline size_t gemm_slot_bytes(const GemmPlan& p, long long M, long long N) {
    return p.splits > 1 ? (size_t)p.splits * (size_t)M * (size_t)((N + 7) / 8 * 8) * 4 : 0;
}

// y = residual + dropout(act(z + bias)), z rounded to fp16 into saved
struct LinearEpilogue {
    const float* bias;                   // or null
    const void* residual;                // bf16, or null
    void* y;                             // bf16
    void* saved;                         // fp16, or null
    int act;
    Dropout drop;
    long long M;
    int N;
    bool vec;                            // rows of y, residual, saved are 16-byte aligned
};
// out = prev + v as bf16 or float; row r goes to row_map[r] (those < 0 nowhere)
struct StoreEpilogue {
    void* out;
    const float* prev;                   // same pitch, or null
    const int* row_map;                  // or null
    long long ld;
    long long split_stride;              // elements between the results of two splits
    long long M;
    int N;
    bool bf16, vec;
};
// Scores h = v + bias of a tile row -> their maximum m and S = sum 2^15 e^{h - m} (stats[row * tiles_n + tile]), the label's score, and, where kept is
// not null, 2^15 e^{h - m} as fp16.
struct CeEpilogue {
    const float* bias;
    int V;
    const int* label;
    float* label_score;
    float2* stats;
    int tiles_n;
    void* kept;
    long long pitch;                     // elements of a row of kept
};
// k-contiguous A, k-slow B
hipError_t launch_linear_gemm(const GemmJob& g, const GemmPlan& p, float* slots, const LinearEpilogue& e, hipStream_t stream);
hipError_t launch_ce_gemm(const GemmJob& g, int tile, const CeEpilogue& e, hipStream_t stream);
// A and B k-contiguous, or both k-slow
hipError_t launch_store_gemm(bool k_slow, const GemmJob& g, const GemmPlan& p, float* slots, const StoreEpilogue& e, hipStream_t stream);

// ---- passes over memory --------------------------------------------------------------------------------------------
// dst[rows_to, ld_to] = src[rows, cols] (dense) from row r0 on, zeros elsewhere; element size 2 or 4
hipError_t launch_pad(const void* src, int size, long long rows, long long cols, long long r0, void* dst, long long rows_to, long long ld_to,
                      hipStream_t stream);

// dz = dy act'(z) mask / (1 - p) into dz [rows_to, ld] (zeros beyond [M, N]; null: not stored), column sums of blocks of SUM_ROWS rows into part
// [ceil(M / SUM_ROWS), ld] (null: none).  bf16: saved fp16, dz bf16; else both float.
constexpr int SUM_ROWS = 128;
struct DzArgs {
    const void* dy;
    const void* saved;
    void* dz;
    float* part;
    long long M, rows_to;
    int N;
    long long ld;
    int act;
    Dropout drop;
    bool vec;
};
hipError_t launch_dz(bool bf16, const DzArgs& a, hipStream_t stream);
// out[n] = prev[n] + sum of part[0 .. blocks) [n]; blocks from *count (rows - row0) where count is not null.  out bf16 or float
hipError_t launch_sum_parts(const float* part, int blocks, long long ld, int N, const int* count, long long row0, const float* prev, void* out,
                            bool bf16, hipStream_t stream);
// fp32: z (pitch ld; may be saved or y) + bias -> saved (or null), y = residual + dropout(act(z + bias)); all but z dense [M, N]
hipError_t launch_linear_rows_f32(const float* z, long long ld, const float* bias, const float* residual, float* y, float* saved, long long M, int N,
                                  int act, const Dropout& drop, hipStream_t stream);
// dst [rows, N] (+)= src (pitch ld)
hipError_t launch_crop_f32(const float* src, long long ld, float* dst, long long rows, int N, bool add, hipStream_t stream);

// ---- cross entropy ---------------------------------------------------------------------------------------------------
// Rows whose label is not `ignore`, in order: their number, places, labels, weights.  Arrays of `cap` entries (a multiple of 256).
struct CeRows {
    int* count;                          // [1]
    int* index;                          // -1 behind the last
    int* label;
    float* weight;
    int* place;                          // [R]: of each row in the order, or -1
};
hipError_t launch_ce_rows(const int* labels, const float* weight, long long R, int ignore, long long cap, const CeRows& r, hipStream_t stream);
// x's rows in that order into xp [.., ld] (zeros beyond D and in the rows behind the last up to fill_to, 0: up to a multiple of 256); loss and dx
// (null: no gradients) of the other rows = 0
hipError_t launch_ce_gather(const void* x, int size, long long R, int D, const CeRows& r, void* xp, long long ld, long long fill_to, float* loss, void* dx,
                            hipStream_t stream);
// per row of a chunk: loss[index], and stats[..].x = factor that turns kept exponentials into weight * probability
hipError_t launch_ce_finish(const CeRows& r, long long row0, long long rows, const float* label_score, float2* stats, int tiles_n, int V, float* loss,
                            bool grads, hipStream_t stream);
// kept -> score gradients bf16, in place; their column sums
hipError_t launch_ce_grad(const CeRows& r, long long row0, long long rows, void* kept, long long pitch, const float2* stats, int tiles_n, int tile, int V,
                          float* part, hipStream_t stream);
// fp32: scores [rows, V] (pitch ld, without the bias) -> loss and, with grads, score gradients in place (zeros in rows behind the last)
hipError_t launch_ce_rows_f32(const CeRows& r, long long row0, long long rows, float* scores, long long ld, int V, const float* b, float* loss,
                              bool grads, hipStream_t stream);
hipError_t launch_col_sums_f32(const float* x, long long rows, long long ld, int N, float* part, hipStream_t stream);
// dx[index[row0 + i]] = src[i] (fp32, D columns of pitch ld)
hipError_t launch_scatter_f32(const CeRows& r, long long row0, long long rows, const float* src, long long ld, int D, float* dx, hipStream_t stream);

}  // namespace rnnt
