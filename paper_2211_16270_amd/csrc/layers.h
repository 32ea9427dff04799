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

// float or bfloat16, or none (p null: zeros)
struct Bias {
    const void* p;
    bool bf16;
#ifdef __HIPCC__
    __device__ __forceinline__ float at(int n) const {
        return p == nullptr ? 0.0f : bf16 ? (float)((const __bf16*)p)[n] : ((const float*)p)[n];
    }
#endif
};

// ---- bf16 matrix products ---------------------------------------------------------------------------------------------
// fp32 products: an fp32 value is the exact sum of three bf16 values, each the rounded rest of the ones before: x = h + m + l with |m| <= 2^-9 |x|, |l| <= 2^-18
// |x|.  A matrix lies as four arrays of its shape, `part` elements apart: h, h where x is finite (else 0), m, l (0 where it is not).  A product
// takes six pairs per 64 of k, the small ones first: h l, m m, l h, h m, m h, h h; what is left out is below 2^-26 of it.  Only the last takes the h that
// may be infinite or NaN, so that those count as what they are.  (Below 2^-110 a value loses what lies under 2^-134.)
constexpr int PARTS = 4, PAIRS = 6;
struct GemmOperand {
    const void* p;
    long long ld;                        // elements
    long long part;
    const void* tail;                    // k-slow operands whose K is no multiple of 64: the last stage's 64 rows, zeros from K on; else null
    int tail_stage;
    int wrap;                            // bf16: stages from here on are those from 0 on again, `part` elements further; 0: none
};
// C[m, n] = sum_k A(m, k) B(k, n); a k-slow operand's extent along the other index is a multiple of 8, a k-contiguous one's K a multiple of 64.
// limit: a count of rows that only the device knows, n = max(0, min(*count - row0, extent)): it bounds M (GEMM_ROWS_M) or K (GEMM_ROWS_K, the operands
// being zero from there to the next multiple of 64).
enum GemmLimit { GEMM_FIXED = 0, GEMM_ROWS_M, GEMM_ROWS_K };
struct GemmJob {
    GemmOperand A, B;
    long long M, N;                      // tiles cover them; operands may be read up to a_rows, b_rows along their other index
    long long a_rows, b_rows;
    int per_block;                       // stages per 64 of k: 1, fp32 products: PAIRS
    int stages;                          // ceil(K / 64) per_block
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
    Bias bias;
    const void* residual;                // bf16, or null
    void* y;                             // bf16
    void* saved;                         // fp16, or null
    int act;
    Dropout drop;
    unsigned long long* rng_used;        // drop.state as the kernels saw it, or null
    long long M;
    int N;
};
// out = prev + scale *unit v as bf16 or float; row r goes to row_map[r] (those < 0 nowhere)
struct StoreEpilogue {
    void* out;
    const float* prev;                   // same pitch, or null
    float scale;
    const float* unit;                   // or null: 1
    const int* row_map;                  // or null
    long long ld;
    long long split_stride;              // elements between the results of two splits
    Bias bias;
    long long M;
    int N;
    bool bf16;
};
// The same in fp32: residual, y, saved float
struct LinearEpilogue32 : LinearEpilogue {};
// Scores h = v + bias of a tile row -> their maximum m and S = sum 2^15 e^{h - m} (stats[row * tiles_n + tile]), the label's score, and, where kept is
// not null, 2^15 e^{h - m} as fp16.
struct CeEpilogue {
    Bias bias;
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
hipError_t launch_linear_gemm(const GemmJob& g, const GemmPlan& p, float* slots, const LinearEpilogue32& e, hipStream_t stream);
hipError_t launch_ce_gemm(const GemmJob& g, int tile, const CeEpilogue& e, hipStream_t stream);
// scores in fp32 (out: float, with the bias)
hipError_t launch_scores_f32(const GemmJob& g, int tile, const StoreEpilogue& e, hipStream_t stream);
// The same two for at most FEW_ROWS rows, x [M, K] and W [K, N] dense, of any size and alignment; the statistics are of parts of FEW_TILE columns.
constexpr int FEW_ROWS = 64, FEW_TILE = 32;
struct FewJob {
    const void* x;
    const void* W;
    int M, K, N;
    bool f32;                            // (results of the fp32 matrix instruction)
};
int few_splits(bool f32, long long M, int K, int N);
hipError_t launch_few_linear(const FewJob& j, int splits, float* slots, const LinearEpilogue& e, hipStream_t stream);
// the epilogue on the sum of slots [splits][M][N up to 8]
hipError_t launch_linear_reduce(bool f32, long long M, int N, int splits, const float* slots, const LinearEpilogue& e, hipStream_t stream);
hipError_t launch_few_ce(const FewJob& j, const CeEpilogue& e, hipStream_t stream);
// The two gradients' products, dx (operands k-contiguous) and dW (operands k-slow), in one launch; then, in another, what remains: the sums of their splits
// and the bias gradient's out of column sums.
struct GradGemm {
    GemmJob g;                           // M = 0: none
    int splits, per_split;
    float* slots;
    StoreEpilogue e;
};
struct PairPlan {
    int tile;
    GemmPlan dx, dw;
};
// small: 128 x 128 tiles only (an operand in two values, GemmOperand::wrap)
PairPlan plan_pair(long long Mx, long long Nx, int stages_x, long long Mw, long long Nw, int stages_w, size_t slot_cap, bool small);
struct SumJob {
    const float* part;
    long long rows, ld;                  // the rows that left the column sums (0: part is not read)
    int N;
    const int* count;                    // of them those below *count - row0, or null
    long long row0;
    const float* prev;
    void* out;                           // null: none
    bool bf16;
    float scale;                         // out = prev + scale *unit times the sum
    const float* unit;                   // or null: 1
};
// parts: fp32 products
hipError_t launch_grad_gemms(bool parts, int tile, const GradGemm& dx, const GradGemm& dw, const SumJob& db, hipStream_t stream);

// ---- passes over memory --------------------------------------------------------------------------------------------
// dst[rows_to, ld_to] = src[rows, cols] (dense) from row r0 on, zeros elsewhere, ld_to a multiple of 8: a copy of 16-bit values, of 32-bit ones, or of floats as
// parts.  Up to three in a launch of their own or behind another kernel's work (`pads` there).
enum PadKind { PAD_NONE = 0, PAD_16, PAD_32, PAD_PARTS };
struct PadJob {
    int kind;
    const void* src;
    long long rows, cols, r0;
    void* dst;
    long long rows_to, ld_to;
};
struct PadJobs {
    PadJob job[3];
    int n;
    void add(int kind, const void* src, long long rows, long long cols, long long r0, void* dst, long long rows_to, long long ld_to) {
        job[n++] = PadJob{kind, src, rows, cols, r0, dst, rows_to, ld_to};
    }
};
hipError_t launch_pads(const PadJobs& j, hipStream_t stream);
// {seed, offset} of a call that launches nothing else
hipError_t launch_pass_rng(const unsigned long long* state, unsigned long long* used, hipStream_t stream);

// Rows per workgroup of a pass over [rows, cols] that leaves column sums, and so per row of these partial sums: 128 where there are workgroups of
// 128 x 256 enough, fewer for a small array (1632 x 640 in fp32, dz: 29.6 us with 128, 39 workgroups).
inline int sum_rows(long long rows, long long cols) {
    int r = 128;
    while (r > 16 && (rows + r - 1) / r * ((cols + 255) / 256) < 1024) r /= 2;
    return r;
}
inline long long sum_blocks(long long rows, long long cols) { return (rows + sum_rows(rows, cols) - 1) / sum_rows(rows, cols); }
// at least sum_blocks(r, cols) for every r <= rows (fewer rows per block below 128 means fewer than 1024 workgroups with twice as many)
inline long long sum_capacity(long long rows, long long cols) {
    const long long few = 2048 / ((cols + 255) / 256) + 2, many = (rows + 127) / 128, most = (rows + 15) / 16;
    return few > many ? (few < most ? few : most) : many;
}
// dz = dy act'(z) mask into dz [rows_to, ld] (zeros beyond [M, N]; null: not stored), column sums of blocks of sum_rows(M, N) rows into part
// [sum_blocks(M, N), ld] (null: none).  bf16: saved fp16, dz bf16; else dy and saved float, dz as parts.  Dropout's 1 / (1 - p) is left to the products'
// epilogue: without it dz of no activation or of relu is dy or 0, and its rounding to bf16 costs nothing.
// rest (bf16, elements): what the rounding left goes there behind dz, as bf16 too; 0: nowhere.
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
    long long rest;
};
hipError_t launch_dz(bool bf16, const DzArgs& a, const PadJobs& pads, hipStream_t stream);
// ---- cross entropy ---------------------------------------------------------------------------------------------------
// Rows whose label is not `ignore`, in order: their number, places, labels, weights.  Arrays of `cap` entries (a multiple of 256).
struct CeRows {
    int* count;                          // [1]; behind it the unit of the score gradients (ce_unit), a float
    int* index;                          // -1 behind the last
    int* label;
    float* weight;
};
#ifdef __HIPCC__
__host__ __device__
#endif
inline const float* ce_unit(const CeRows& r) { return reinterpret_cast<const float*>(r.count + 1); }
// x's rows in that order into xp [.., ld] (zeros beyond D and in the rows behind the last up to a multiple of 256; f32: as parts of cap rows); loss and dx
// (null: no gradients) of the other rows = 0.  place: scratch of ce_place_ints(cap) ints for more than GATHER_SCAN rows.
constexpr long long GATHER_SCAN = 16384, CE_SCAN_ROWS = 4096;
inline long long ce_place_ints(long long cap) { return cap + 2 * ((cap + CE_SCAN_ROWS - 1) / CE_SCAN_ROWS); }
hipError_t launch_ce_gather(const void* x, bool f32, long long R, int D, const int* labels, const float* weight, int ignore, long long cap, int* place,
                            const CeRows& r, void* xp, long long ld, float* loss, void* dx, const PadJobs& pads, hipStream_t stream);
// Rows [row0, row0 + rows) of that order and the statistics of their scores, tiles_n parts of 2^tile_log2 columns each (arrays: of the chunk)
struct CeChunk {
    CeRows r;
    long long row0, rows;
    const float* label_score;
    const float2* stats;
    int tiles_n, tile_log2, V;
    float4* scale;                       // [rows] {maximum, weight / sum, the label's gradient}: what turns kept exponentials into score gradients
    float* loss;
    bool identity;                       // r.label are the caller's labels, every row is its own place and the ones with `ignore` have loss 0
    int ignore;
};
// loss, scale
hipError_t launch_ce_finish(const CeChunk& c, hipStream_t stream);
// kept -> score gradients over the unit, bf16, in place; their column sums (part: null: none).  Does launch_ce_finish's work too where ce_grad_finishes says so.
// FINISH_LOADS parts for each of the 256 / R threads of a row at most: every column block does it again (777 x 443 x 5001, 40 parts: a launch of 4 us less; 128 parts with
// R = 128 would be 64 loads a thread in 128 column blocks).
constexpr int FINISH_LOADS = 8;
inline bool ce_grad_finishes(long long rows, long long V, int tiles_n) { return (long long)tiles_n * sum_rows(rows, V) <= FINISH_LOADS * 256; }
// rest: as in DzArgs
hipError_t launch_ce_grad(const CeChunk& c, void* kept, long long pitch, long long rest, float* part, hipStream_t stream);
// fp32: scores [rows, V] (pitch ld) of a chunk -> loss and, where grad is not null, the score gradients as parts (`rows` rows of pitch ld; zeros behind the
// last up to a multiple of 64)
hipError_t launch_ce_rows_f32(const CeRows& r, long long row0, long long rows, const float* scores, long long ld, int V, float* loss, void* grad,
                              hipStream_t stream);
// total = sum of weight[r] loss[r] over the rows whose weight is not 0 (null: ones)
hipError_t launch_ce_total(const float* loss, const float* weight, long long R, float* total, hipStream_t stream);
// three arrays (those of length 0: none) times *factor, in place; a factor of 1 moves nothing
hipError_t launch_scale(const float* factor, void* const (&p)[3], const long long (&n)[3], const bool (&bf16)[3], hipStream_t stream);
// column sums of parts [rows, ld], of the rows below *count - row0
hipError_t launch_col_sums_f32(const void* x, long long rows, long long ld, int N, const int* count, long long row0, float* part, hipStream_t stream);
}  // namespace rnnt
