// C-ABI entry points of include/rnnt_layers.h: argument checks, workspace layouts and launch sequences.  Compiled with hipcc as host code.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "../../include/rnnt_layers.h"
#include "kernels.h"
#include "layers.h"

using namespace rnnt;

namespace {

#define LAYER_HIP(expr)                              \
    do {                                             \
        const hipError_t e_ = (expr);                \
        if (e_ != hipSuccess) {                      \
            note_hip_error(e_, "layers.cpp", __LINE__); \
            (void)hipGetLastError();                 \
            return RNNT_ERR_HIP;                     \
        }                                            \
    } while (0)

constexpr int64_t MAX_ROWS = 1 << 30;
constexpr int32_t MAX_WIDTH = 1 << 20;
constexpr size_t SLOT_CAP = 256u << 20;               // bytes of partial sums per product
constexpr size_t CE_CHUNK = 1u << 30;                 // default bytes of a chunk's exponentials or scores

long long up(long long x, long long a) { return (x + a - 1) / a * a; }

bool aligned(std::initializer_list<const void*> ptrs) {
    for (const void* p : ptrs)
        if ((uintptr_t)p % 16 != 0) return false;
    return true;
}

// Parts of a workspace, each on a 256-byte boundary
struct Carver {
    size_t bytes = 0;
    size_t take(size_t n) {
        const size_t at = bytes;
        bytes += (n + 255) / 256 * 256;
        return at;
    }
};
bool workspace_ok(const void* ws, size_t have, size_t need) { return need == 0 || (ws != nullptr && (uintptr_t)ws % 256 == 0 && have >= need); }

// fp32 products: two workgroups of 128 x 128 per compute unit, so a sum over k is cut into as many parts as make 512 of them, each at least 64 deep
// (2048 x 512 out of a depth of 4096: 180 us in one part, 64 workgroups); at most 16384 deep, so that its rounding does not grow with it.  Parts are
// stored apart and added in order.
int splits_f32(long long M, long long N, long long K) {
    const double tiles = (double)((M + 127) / 128) * (double)((N + 127) / 128);
    long long s = tiles >= 512.0 ? 1 : (long long)(512.0 / std::max(1.0, tiles));
    s = std::min(s, std::max(1LL, K / 64));
    while (s > 1 && (double)s * (double)M * (double)N * 4.0 > (double)SLOT_CAP) --s;
    s = std::max(s, (K + 16383) / 16384);
    return K > 0 ? gemm_f32_split_count(K, (int)s) : 1;
}
size_t slots_f32(int splits, long long rows, long long ld) { return (size_t)splits * (size_t)rows * (size_t)ld * 4; }

// ---- linear -------------------------------------------------------------------------------------------------------------
rnnt_status check_linear(const rnnt_linear_desc* d, bool backward) {
    if (!d) return RNNT_ERR_NULL;
    if (d->M < 0 || d->M > MAX_ROWS || d->K < 1 || d->K > MAX_WIDTH || d->N < 1 || d->N > MAX_WIDTH) return RNNT_ERR_SHAPE;
    if (d->dtype != RNNT_F32 && d->dtype != RNNT_BF16) return RNNT_ERR_UNSUPPORTED;
    if (d->activation < 0 || d->activation >= ACT_COUNT) return RNNT_ERR_UNSUPPORTED;
    if (!(d->dropout >= 0.0f && d->dropout < 1.0f) || d->bias_bf16 < 0 || d->bias_bf16 > 1) return RNNT_ERR_SHAPE;
    if (backward) {
        if (d->accumulate_params < 0 || d->accumulate_params > 1 || d->param_grads_bf16 < 0 || d->param_grads_bf16 > 3) return RNNT_ERR_SHAPE;
        if (d->param_grads_bf16 != 0 && (d->dtype != RNNT_BF16 || d->accumulate_params)) return RNNT_ERR_UNSUPPORTED;
    }
    return RNNT_OK;
}
unsigned dropout_cut(float p) { return (unsigned)std::min(65535.0, std::nearbyint((double)p * 65536.0)); }
Dropout make_dropout(const rnnt_linear_desc& d, const uint64_t* rng) {
    const unsigned cut = dropout_cut(d.dropout);
    return Dropout{(const unsigned long long*)rng, cut, (float)(65536.0 / (65536.0 - cut))};
}

// Where the operands of the products lie.  bf16: rows of 64 elements' multiples along a contiguous contraction, 8 along the other index, else a padded copy.
struct LinearPlan {
    bool bf16, backward;
    bool few;                             // forward pass of at most FEW_ROWS rows: one launch on the arrays as they are
    int few_splits;
    bool copy_x, copy_w, own_dz;
    long long Kp, Np, Mp;                 // pitches of the copies and of dz; rows of dz
    size_t off_x, off_w, off_dz, off_xt, off_dyt, off_part, off_slots, off_slots_w, bytes;
    GemmPlan y;
    PairPlan grads;
    int y32, dx32, dw32;                  // fp32: parts of the three sums
};
LinearPlan plan_linear(const rnnt_linear_desc& d, bool backward) {
    LinearPlan p{};
    p.bf16 = d.dtype == RNNT_BF16;
    p.backward = backward;
    const long long M = d.M, K = d.K, N = d.N;
    const size_t e = p.bf16 ? 2 : 4;
    Carver c;
    const bool plain = d.activation == ACT_NONE && dropout_cut(d.dropout) == 0;
    if (p.bf16) {
        p.Kp = up(K, 64);
        p.Np = up(N, 64);
        p.Mp = up(M, 64);
        if (!backward && M <= FEW_ROWS) {
            p.few = true;
            p.few_splits = few_splits(M, d.K, d.N);
            p.off_slots = c.take(p.few_splits > 1 ? (size_t)p.few_splits * M * up(N, 8) * 4 : 0);
        } else if (!backward) {
            p.copy_x = K % 64 != 0;
            p.copy_w = K % 64 != 0 || N % 8 != 0;
            p.y = plan_gemm(M, N, (int)(p.Kp / 64), SLOT_CAP);
            p.off_x = c.take(p.copy_x ? (size_t)M * p.Kp * 2 : 0);
            p.off_w = c.take(p.copy_w ? (size_t)p.Kp * p.Np * 2 : 0);
            p.off_slots = c.take(gemm_slot_bytes(p.y, M, N));
        } else {
            p.own_dz = !plain || N % 64 != 0;
            p.copy_x = K % 8 != 0;
            p.copy_w = N % 64 != 0;
            p.grads = plan_pair(M, K, (int)(p.Np / 64), K, N, (int)(p.Mp / 64), SLOT_CAP);
            p.off_dz = c.take(p.own_dz ? (size_t)p.Mp * p.Np * 2 : 0);
            p.off_x = c.take(p.copy_x ? (size_t)p.Mp * p.Kp * 2 : 0);
            p.off_w = c.take(p.copy_w ? (size_t)K * p.Np * 2 : 0);
            p.off_xt = c.take(!p.copy_x && M % 64 != 0 ? (size_t)64 * K * 2 : 0);
            p.off_dyt = c.take(!p.own_dz && M % 64 != 0 ? (size_t)64 * N * 2 : 0);
            p.off_part = c.take((size_t)sum_capacity(M, N) * p.Np * 4);
            p.off_slots = c.take(gemm_slot_bytes(p.grads.dx, M, K));
            p.off_slots_w = c.take(gemm_slot_bytes(p.grads.dw, K, N));
        }
    } else {
        p.Kp = up(K, 4);
        p.Np = up(N, 4);
        p.copy_x = K % 4 != 0;
        p.copy_w = K % 4 != 0 || N % 4 != 0;
        p.off_x = c.take(p.copy_x ? (size_t)M * p.Kp * e : 0);
        p.off_w = c.take(p.copy_w ? (size_t)p.Kp * p.Np * e : 0);
        if (!backward) {
            p.y32 = splits_f32(M, p.Np, p.Kp);
            p.off_slots = c.take(p.y32 > 1 || N % 4 != 0 ? slots_f32(p.y32, M, p.Np) : 0);
        } else {
            p.own_dz = !plain || N % 4 != 0;
            p.off_dz = c.take(p.own_dz ? (size_t)M * p.Np * e : 0);
            p.off_part = c.take((size_t)sum_capacity(M, N) * p.Np * 4);
            p.dx32 = splits_f32(M, K, p.Np);
            p.dw32 = splits_f32(p.Kp, p.Np, M);
            p.off_slots = c.take(std::max(p.dx32 > 1 ? slots_f32(p.dx32, M, K) : 0, slots_f32(p.dw32, p.Kp, p.Np)));
        }
    }
    p.bytes = c.bytes;
    return p;
}

rnnt_status linear_fwd_bf16(const rnnt_linear_desc& d, const LinearPlan& p, const void* x, const void* W, const Bias& b, const void* residual,
                            const Dropout& drop, uint64_t* rng_used, void* y, void* saved, unsigned char* ws, hipStream_t stream) {
    const long long M = d.M, K = d.K, N = d.N;
    const LinearEpilogue e{b, residual, y, saved, d.activation, drop, (unsigned long long*)rng_used, M, d.N};
    if (p.few) {
        LAYER_HIP(launch_few_linear(FewJob{x, W, (int)M, d.K, d.N}, p.few_splits, (float*)(ws + p.off_slots), e, stream));
        return RNNT_OK;
    }
    if (p.copy_x) LAYER_HIP(launch_pad(x, 2, M, K, 0, ws + p.off_x, M, p.Kp, stream));
    if (p.copy_w) LAYER_HIP(launch_pad(W, 2, K, N, 0, ws + p.off_w, p.Kp, p.Np, stream));
    GemmJob g{};
    g.A = GemmOperand{p.copy_x ? ws + p.off_x : x, p.copy_x ? p.Kp : K, nullptr, -1};
    g.B = GemmOperand{p.copy_w ? ws + p.off_w : W, p.copy_w ? p.Np : N, nullptr, -1};
    g.M = g.a_rows = M;
    g.N = N;
    g.b_rows = p.copy_w ? p.Np : N;
    g.stages = (int)(p.Kp / 64);
    LAYER_HIP(launch_linear_gemm(g, p.y, (float*)(ws + p.off_slots), e, stream));
    return RNNT_OK;
}

rnnt_status linear_bwd_bf16(const rnnt_linear_desc& d, const LinearPlan& p, const void* x, const void* W, const void* saved, const Dropout& drop,
                            const void* dy, void* dx, void* dW, void* db, unsigned char* ws, hipStream_t stream) {
    const long long M = d.M, K = d.K, N = d.N;
    float* part = (float*)(ws + p.off_part);
    if (M > 0 && (db || (p.own_dz && (dx || dW)))) {
        const DzArgs a{dy, d.activation == ACT_NONE ? nullptr : saved, p.own_dz && (dx || dW) ? ws + p.off_dz : nullptr, db ? part : nullptr, M,
                       p.own_dz ? p.Mp : M, d.N, p.Np, d.activation, drop};
        LAYER_HIP(launch_dz(true, a, stream));
    }
    const void* dz = p.own_dz ? ws + p.off_dz : dy;
    const long long ld_dz = p.own_dz ? p.Np : N;
    GradGemm gx{}, gw{};
    if (dx && M > 0) {
        if (p.copy_w) LAYER_HIP(launch_pad(W, 2, K, N, 0, ws + p.off_w, K, p.Np, stream));
        gx.g.A = GemmOperand{dz, ld_dz, nullptr, -1};
        gx.g.B = GemmOperand{p.copy_w ? ws + p.off_w : W, p.copy_w ? p.Np : N, nullptr, -1};
        gx.g.M = gx.g.a_rows = M;
        gx.g.N = gx.g.b_rows = K;
        gx.g.stages = (int)(p.Np / 64);
        gx.splits = p.grads.dx.splits;
        gx.per_split = p.grads.dx.per_split;
        gx.slots = (float*)(ws + p.off_slots);
        gx.e = StoreEpilogue{dx, nullptr, nullptr, K, 0, M, d.K, true};
    }
    if (dW) {
        const bool ragged = M % 64 != 0;
        const long long whole = M / 64 * 64;
        if (p.copy_x) LAYER_HIP(launch_pad(x, 2, M, K, 0, ws + p.off_x, p.Mp, p.Kp, stream));
        else if (ragged) LAYER_HIP(launch_pad(x, 2, M, K, whole, ws + p.off_xt, 64, K, stream));
        if (!p.own_dz && ragged) LAYER_HIP(launch_pad(dy, 2, M, N, whole, ws + p.off_dyt, 64, N, stream));
        gw.g.A = GemmOperand{p.copy_x ? ws + p.off_x : x, p.copy_x ? p.Kp : K, !p.copy_x && ragged ? ws + p.off_xt : nullptr, (int)(whole / 64)};
        gw.g.B = GemmOperand{dz, ld_dz, !p.own_dz && ragged ? ws + p.off_dyt : nullptr, (int)(whole / 64)};
        gw.g.M = K;
        gw.g.a_rows = p.copy_x ? p.Kp : K;
        gw.g.N = N;
        gw.g.b_rows = ld_dz;
        gw.g.stages = (int)(p.Mp / 64);
        gw.splits = p.grads.dw.splits;
        gw.per_split = p.grads.dw.per_split;
        gw.slots = (float*)(ws + p.off_slots_w);
        gw.e = StoreEpilogue{dW, d.accumulate_params ? (const float*)dW : nullptr, nullptr, N, 0, K, d.N, (d.param_grads_bf16 & 1) != 0};
    }
    const SumJob sum{db ? part : nullptr, M, p.Np, d.N, nullptr, 0, d.accumulate_params ? (const float*)db : nullptr, db, (d.param_grads_bf16 & 2) != 0};
    LAYER_HIP(launch_grad_gemms(p.grads.tile, gx, gw, sum, stream));
    return RNNT_OK;
}

rnnt_status linear_fwd_f32(const rnnt_linear_desc& d, const LinearPlan& p, const float* x, const float* W, const Bias& b, const float* residual,
                           const Dropout& drop, uint64_t* rng_used, float* y, float* saved, unsigned char* ws, hipStream_t stream) {
    const long long M = d.M, K = d.K, N = d.N;
    if (p.copy_x) LAYER_HIP(launch_pad(x, 4, M, K, 0, ws + p.off_x, M, p.Kp, stream));
    if (p.copy_w) LAYER_HIP(launch_pad(W, 4, K, N, 0, ws + p.off_w, p.Kp, p.Np, stream));
    float* z = p.y32 > 1 || N % 4 != 0 ? (float*)(ws + p.off_slots) : saved ? saved : y;
    LAYER_HIP(launch_gemm_f32_split(0, 1, p.copy_x ? (const float*)(ws + p.off_x) : x, p.Kp, p.copy_w ? (const float*)(ws + p.off_w) : W, p.Np, z, p.Np, M,
                                    p.Np, p.Kp, p.y32, M * p.Np, stream));
    LAYER_HIP(launch_linear_rows_f32(z, p.Np, p.y32, M * p.Np, b, residual, y, saved, M, d.N, d.activation, drop,
                                     (unsigned long long*)rng_used, stream));
    return RNNT_OK;
}

rnnt_status linear_bwd_f32(const rnnt_linear_desc& d, const LinearPlan& p, const float* x, const float* W, const float* saved, const Dropout& drop,
                           const float* dy, float* dx, float* dW, float* db, unsigned char* ws, hipStream_t stream) {
    const long long M = d.M, K = d.K, N = d.N;
    float* part = (float*)(ws + p.off_part);
    if (M > 0 && (db || (p.own_dz && (dx || dW)))) {
        const DzArgs a{dy, d.activation == ACT_NONE ? nullptr : saved, p.own_dz && (dx || dW) ? ws + p.off_dz : nullptr, db ? part : nullptr, M, M, d.N, p.Np,
                       d.activation, drop};
        LAYER_HIP(launch_dz(false, a, stream));
    }
    if (db)
        LAYER_HIP(launch_sum_parts(SumJob{part, M, p.Np, d.N, nullptr, 0, d.accumulate_params ? db : nullptr, db, false}, stream));
    const float* dz = p.own_dz ? (const float*)(ws + p.off_dz) : dy;
    if (p.copy_w && dx && M > 0) LAYER_HIP(launch_pad(W, 4, K, N, 0, ws + p.off_w, p.Kp, p.Np, stream));
    float* slots = (float*)(ws + p.off_slots);
    if (dx && M > 0) {
        LAYER_HIP(launch_gemm_f32_split(0, 0, dz, p.Np, p.copy_w ? (const float*)(ws + p.off_w) : W, p.Np, p.dx32 > 1 ? slots : dx, K, M, K, p.Np, p.dx32,
                                        M * K, stream));
        if (p.dx32 > 1) LAYER_HIP(launch_reduce_f32(slots, K, p.dx32, M * K, nullptr, dx, M, d.K, false, stream));
    }
    if (dW && M == 0) {
        if (!d.accumulate_params) LAYER_HIP(launch_pad(nullptr, 4, 0, 0, 0, dW, K, N, stream));
    } else if (dW) {
        if (p.copy_x) LAYER_HIP(launch_pad(x, 4, M, K, 0, ws + p.off_x, M, p.Kp, stream));
        const bool direct = p.dw32 == 1 && !p.copy_w && !d.accumulate_params;
        LAYER_HIP(launch_gemm_f32_split(1, 1, p.copy_x ? (const float*)(ws + p.off_x) : x, p.Kp, dz, p.Np, direct ? dW : slots, p.Np, p.Kp, p.Np, M, p.dw32,
                                        p.Kp * p.Np, stream));
        if (!direct) LAYER_HIP(launch_reduce_f32(slots, p.Np, p.dw32, p.Kp * p.Np, nullptr, dW, K, d.N, d.accumulate_params != 0, stream));
    }
    return RNNT_OK;
}

// ---- cross entropy --------------------------------------------------------------------------------------------------------
rnnt_status check_ce(const rnnt_ce_desc* d, bool grads) {
    if (!d) return RNNT_ERR_NULL;
    if (d->R < 0 || d->R > MAX_ROWS || d->D < 1 || d->D > MAX_WIDTH || d->V < 1 || d->V > MAX_WIDTH) return RNNT_ERR_SHAPE;
    if (d->bias_bf16 < 0 || d->bias_bf16 > 1) return RNNT_ERR_SHAPE;
    if (d->dtype != RNNT_F32 && d->dtype != RNNT_BF16) return RNNT_ERR_UNSUPPORTED;
    if (grads) {
        if (d->accumulate_params < 0 || d->accumulate_params > 1 || d->param_grads_bf16 < 0 || d->param_grads_bf16 > 3) return RNNT_ERR_SHAPE;
        if (d->param_grads_bf16 != 0 && (d->dtype != RNNT_BF16 || d->accumulate_params)) return RNNT_ERR_UNSUPPORTED;
    }
    return RNNT_OK;
}

struct CePlan {
    bool bf16, grads, copy_w;
    bool few;                             // at most FEW_ROWS rows: scores by one launch on W as it is
    bool identity;                        // ... and without gradients on x as it is
    long long cap, chunk, Dp, Vp, pitch;  // rows (a multiple of 256) in all and per chunk; padded widths; elements of a chunk row
    int chunks, tile, tile_log2, tiles_n;
    size_t off_count, off_index, off_label, off_weight, off_place, off_x, off_w, off_chunk, off_score, off_stats, off_scale, off_part, off_slots, off_slots_w, off_acc,
        off_dbacc, bytes;
    PairPlan pair;
    int dx32, dw32;                       // fp32: parts of the gradients' sums
};
CePlan plan_ce_chunk(const rnnt_ce_desc& d, bool grads, long long chunk) {
    CePlan p{};
    p.bf16 = d.dtype == RNNT_BF16;
    p.grads = grads;
    const long long R = d.R, D = d.D, V = d.V;
    p.cap = std::max(256LL, up(R, 256));
    p.chunk = std::min(chunk, p.cap);
    p.chunks = (int)((p.cap + p.chunk - 1) / p.chunk);
    const size_t e = p.bf16 ? 2 : 4;
    p.Dp = up(D, p.bf16 ? 64 : 4);
    p.Vp = up(V, p.bf16 ? 64 : 4);
    p.copy_w = p.Dp != D || p.Vp != V;
    p.few = p.bf16 && R <= FEW_ROWS;
    p.identity = p.few && !grads;
    Carver c;
    if (p.identity) {
        p.copy_w = false;
        p.tile = FEW_TILE;
        p.tile_log2 = 5;
        p.tiles_n = (int)((V + FEW_TILE - 1) / FEW_TILE);
        p.off_score = c.take((size_t)FEW_ROWS * 4);
        p.off_stats = c.take((size_t)R * p.tiles_n * 8);
        p.bytes = c.bytes;
        return p;
    }
    p.off_count = c.take(4);
    p.off_index = c.take((size_t)p.cap * 4);
    p.off_label = c.take((size_t)p.cap * 4);
    p.off_weight = c.take((size_t)p.cap * 4);
    p.off_place = c.take(R > GATHER_SCAN ? (size_t)p.cap * 4 : 0);
    p.off_x = c.take((size_t)p.cap * p.Dp * e);
    p.off_w = c.take(p.copy_w ? (size_t)p.Dp * p.Vp * e : 0);
    if (p.bf16) {
        // (a row is 128 bytes longer than whole tiles: rows of a power-of-two length would all start in the same memory channel)
        p.pitch = up(V, 256) + 64;
        p.tile = p.few ? FEW_TILE : plan_gemm(p.chunk, V, (int)(p.Dp / 64), 0).tile;
        p.tile_log2 = p.few ? 5 : p.tile == 256 ? 8 : 7;
        // (few: the columns of zeros up to Vp have parts of their own)
        p.tiles_n = (int)(((p.few ? p.Vp : V) + p.tile - 1) / p.tile);
        p.off_score = c.take((size_t)p.chunk * 4);
        p.off_stats = c.take((size_t)p.chunk * p.tiles_n * 8);
        p.off_scale = c.take((size_t)p.chunk * 8);
        if (grads) {
            p.off_chunk = c.take((size_t)p.chunk * p.pitch * 2);
            p.off_part = c.take((size_t)sum_capacity(p.chunk, V) * p.pitch * 4);
            p.pair = plan_pair(p.chunk, D, (int)(p.Vp / 64), D, V, (int)(p.chunk / 64), SLOT_CAP);
            p.off_slots = c.take(gemm_slot_bytes(p.pair.dx, p.chunk, D));
            p.off_slots_w = c.take(gemm_slot_bytes(p.pair.dw, D, V));
            // the weight gradient's sum over the chunks, where its output is bfloat16
            p.off_acc = c.take(p.chunks > 1 && (d.param_grads_bf16 & 1) ? (size_t)D * V * 4 : 0);
            p.off_dbacc = c.take(p.chunks > 1 ? (size_t)V * 4 : 0);
        }
    } else {
        p.pitch = p.Vp;
        p.off_chunk = c.take((size_t)p.chunk * p.pitch * 4);
        if (grads) {
            p.off_part = c.take((size_t)sum_capacity(p.chunk, V) * p.pitch * 4);
            p.dx32 = splits_f32(p.chunk, D, p.Vp);
            p.dw32 = splits_f32(p.Dp, p.Vp, p.chunk);
            p.off_slots = c.take(std::max(slots_f32(p.dx32, p.chunk, D), slots_f32(p.dw32, p.Dp, p.Vp)));
            p.off_dbacc = c.take(p.chunks > 1 ? (size_t)V * 4 : 0);
        }
    }
    p.bytes = c.bytes;
    return p;
}
// The largest chunks whose plan takes at most `budget` bytes (0: whose buffers take at most CE_CHUNK), at least 256 rows
CePlan plan_ce(const rnnt_ce_desc& d, bool grads, size_t budget) {
    const long long all = std::max(256LL, up(d.R, 256));
    const size_t row = d.dtype == RNNT_BF16 ? (size_t)(up(d.V, 256) + 64) * 2 : (size_t)up(d.V, 4) * 4;
    if (budget == 0) {
        // equal chunks
        const long long most = std::max(256LL, (long long)(CE_CHUNK / row) / 256 * 256), n = (all + most - 1) / most;
        return plan_ce_chunk(d, grads, up((all + n - 1) / n, 256));
    }
    long long lo = 1, hi = all / 256;                 // in units of 256 rows; lo always taken
    CePlan best = plan_ce_chunk(d, grads, 256);
    while (lo < hi) {
        const long long mid = (lo + hi + 1) / 2;
        const CePlan p = plan_ce_chunk(d, grads, mid * 256);
        if (p.bytes <= budget) {
            lo = mid;
            best = p;
        } else hi = mid - 1;
    }
    return best;
}

rnnt_status run_ce(const rnnt_ce_desc& d, const CePlan& p, const void* x, const void* W, const void* b_ptr, const int32_t* label, const float* row_weight,
                   float* loss, void* dx, void* dW, void* db, unsigned char* ws, hipStream_t stream) {
    const long long D = d.D, V = d.V;
    const Bias b{b_ptr, d.bias_bf16 != 0};
    const CeRows rows{(int*)(ws + p.off_count), (int*)(ws + p.off_index), (int*)(ws + p.off_label), (float*)(ws + p.off_weight)};
    const int size = p.bf16 ? 2 : 4;
    if (p.identity) {
        if (d.R == 0) return RNNT_OK;
        CeRows own{};
        own.label = const_cast<int*>(label);
        const CeEpilogue e{b, d.V, label, (float*)(ws + p.off_score), (float2*)(ws + p.off_stats), p.tiles_n, nullptr, 0};
        LAYER_HIP(launch_few_ce(FewJob{x, W, (int)d.R, d.D, d.V}, e, stream));
        LAYER_HIP(launch_ce_finish(CeChunk{own, 0, d.R, e.label_score, e.stats, p.tiles_n, p.tile_log2, d.V, nullptr, loss, true, d.ignore_label}, stream));
        return RNNT_OK;
    }
    void* xp = ws + p.off_x;
    if (d.R > 0) {
        LAYER_HIP(launch_ce_gather(x, size, d.R, d.D, label, row_weight, d.ignore_label, p.cap, (int*)(ws + p.off_place), rows, xp, p.Dp,
                                   p.bf16 ? 0 : p.cap, loss, p.grads ? dx : nullptr, stream));
    } else if (!p.grads) return RNNT_OK;
    else LAYER_HIP(launch_pad(nullptr, 4, 0, 0, 0, rows.count, 1, 1, stream));       // (no rows: the gradients of an empty sum)
    if (p.copy_w) LAYER_HIP(launch_pad(W, size, D, V, 0, ws + p.off_w, p.Dp, p.Vp, stream));
    const void* Wu = p.copy_w ? ws + p.off_w : W;
    unsigned char* chunk = ws + p.off_chunk;
    float* part = (float*)(ws + p.off_part);
    for (int k = 0; k < p.chunks; ++k) {
        const long long row0 = (long long)k * p.chunk, n = std::min(p.chunk, p.cap - row0);
        const bool first = k == 0, last = k == p.chunks - 1;
        const unsigned char* xc = (const unsigned char*)xp + (size_t)row0 * p.Dp * size;
        if (p.bf16) {
            GemmJob g{};
            g.A = GemmOperand{xc, p.Dp, nullptr, -1};
            g.B = GemmOperand{Wu, p.Vp, nullptr, -1};
            g.M = g.a_rows = n;
            g.N = V;
            g.b_rows = p.Vp;
            g.stages = (int)(p.Dp / 64);
            g.limit = GEMM_ROWS_M;
            g.count = rows.count;
            g.row0 = row0;
            const CeEpilogue e{b, d.V, rows.label + row0, (float*)(ws + p.off_score), (float2*)(ws + p.off_stats), p.tiles_n,
                               p.grads ? chunk : nullptr, p.pitch};
            const CeChunk c{rows, row0, n, e.label_score, e.stats, p.tiles_n, p.tile_log2, d.V, (float2*)(ws + p.off_scale), loss, false, 0};
            if (d.R > 0) {
                if (p.few) LAYER_HIP(launch_few_ce(FewJob{xc, Wu, (int)d.R, (int)p.Dp, (int)p.Vp}, e, stream));
                else LAYER_HIP(launch_ce_gemm(g, p.tile, e, stream));
                if (!p.grads || !ce_grad_finishes(p.tiles_n)) LAYER_HIP(launch_ce_finish(c, stream));
            }
            if (!p.grads) continue;
            if (d.R > 0) LAYER_HIP(launch_ce_grad(c, chunk, p.pitch, db ? part : nullptr, stream));
            GradGemm gx{}, gw{};
            if (d.R > 0) {
                gx.g = g;
                gx.g.A = GemmOperand{chunk, p.pitch, nullptr, -1};
                gx.g.N = gx.g.b_rows = D;
                gx.g.stages = (int)(p.Vp / 64);
                gx.splits = p.pair.dx.splits;
                gx.per_split = p.pair.dx.per_split;
                gx.slots = (float*)(ws + p.off_slots);
                gx.e = StoreEpilogue{dx, nullptr, rows.index + row0, D, 0, n, d.D, true};
            }
            gw.g.A = GemmOperand{xc, p.Dp, nullptr, -1};
            gw.g.B = GemmOperand{chunk, p.pitch, nullptr, -1};
            gw.g.M = D;
            gw.g.a_rows = p.Dp;
            gw.g.N = V;
            gw.g.b_rows = p.Vp;
            gw.g.stages = (int)(n / 64);
            gw.g.limit = GEMM_ROWS_K;
            gw.g.count = rows.count;
            gw.g.row0 = row0;
            gw.splits = p.pair.dw.splits;
            gw.per_split = p.pair.dw.per_split;
            gw.slots = (float*)(ws + p.off_slots_w);
            const bool w16 = (d.param_grads_bf16 & 1) != 0, b16 = (d.param_grads_bf16 & 2) != 0;
            float* acc = w16 ? (float*)(ws + p.off_acc) : (float*)dW;
            gw.e = StoreEpilogue{last ? dW : acc, !first || d.accumulate_params ? acc : nullptr, nullptr, V, 0, D, d.V, last && w16};
            float* dba = (float*)(ws + p.off_dbacc);
            const SumJob sum{db ? part : nullptr, n, p.pitch, d.V, rows.count, row0, first ? (d.accumulate_params ? (const float*)db : nullptr) : dba,
                             last ? db : (void*)dba, last && b16};
            LAYER_HIP(launch_grad_gemms(p.pair.tile, gx, gw, sum, stream));
        } else {
            float* S = (float*)chunk;
            if (d.R > 0) {
                LAYER_HIP(launch_gemm_f32_split(0, 1, (const float*)xc, p.Dp, (const float*)Wu, p.Vp, S, p.pitch, n, p.Vp, p.Dp, 1, 0, stream));
                LAYER_HIP(launch_ce_rows_f32(rows, row0, n, S, p.pitch, d.V, b, loss, p.grads, stream));
            }
            if (!p.grads) continue;
            if (d.R == 0) {
                if (!d.accumulate_params) LAYER_HIP(launch_pad(nullptr, 4, 0, 0, 0, dW, D, V, stream));
            } else {
                float* slots = (float*)(ws + p.off_slots);
                const int sx = gemm_f32_split_count(p.Vp, p.dx32), sw = gemm_f32_split_count(n, std::min<long long>(p.dw32, std::max(1LL, n / 64)));
                LAYER_HIP(launch_gemm_f32_split(0, 0, S, p.pitch, (const float*)Wu, p.Vp, slots, D, n, D, p.Vp, sx, n * D, stream));
                LAYER_HIP(launch_reduce_f32(slots, D, sx, n * D, rows.index + row0, (float*)dx, n, d.D, false, stream));
                const bool add = !first || d.accumulate_params, direct = sw == 1 && !p.copy_w && !add;
                LAYER_HIP(launch_gemm_f32_split(1, 1, (const float*)xc, p.Dp, S, p.pitch, direct ? (float*)dW : slots, p.Vp, p.Dp, p.Vp, n, sw,
                                                p.Dp * p.Vp, stream));
                if (!direct) LAYER_HIP(launch_reduce_f32(slots, p.Vp, sw, p.Dp * p.Vp, nullptr, (float*)dW, D, d.V, add, stream));
                if (db) LAYER_HIP(launch_col_sums_f32(S, n, p.pitch, d.V, part, stream));
            }
            if (db) {
                float* dba = (float*)(ws + p.off_dbacc);
                LAYER_HIP(launch_sum_parts(SumJob{part, n, p.pitch, d.V, rows.count, row0,
                                                  first ? (d.accumulate_params ? (const float*)db : nullptr) : dba, last ? db : (void*)dba, false},
                                           stream));
            }
        }
    }
    return RNNT_OK;
}

}  // namespace

extern "C" size_t rnnt_linear_workspace_bytes(const rnnt_linear_desc* desc, int32_t backward) {
    if (check_linear(desc, backward != 0) != RNNT_OK) return 0;
    return plan_linear(*desc, backward != 0).bytes;
}

extern "C" rnnt_status rnnt_linear_fwd(const rnnt_linear_desc* desc, const void* x, const void* W, const void* b, const void* residual,
                                       const uint64_t* rng, uint64_t* rng_used, void* y, void* saved, void* workspace, size_t workspace_bytes, void* hip_stream) {
    const rnnt_status st = check_linear(desc, false);
    if (st != RNNT_OK) return st;
    if (!W || (desc->M > 0 && (!x || !y))) return RNNT_ERR_NULL;
    const Dropout drop = make_dropout(*desc, rng);
    if (drop.cut != 0 && !rng) return RNNT_ERR_NULL;
    if (!aligned({x, W, b, residual, y, saved}) || (((uintptr_t)rng | (uintptr_t)rng_used) % 8) != 0) return RNNT_ERR_UNSUPPORTED;
    if (rng_used && !rng) return RNNT_ERR_NULL;
    const LinearPlan p = plan_linear(*desc, false);
    if (!workspace_ok(workspace, workspace_bytes, p.bytes)) return RNNT_ERR_WORKSPACE;
    if (desc->M == 0) return RNNT_OK;
    unsigned char* ws = (unsigned char*)workspace;
    const Bias bias{b, desc->bias_bf16 != 0};
    if (p.bf16) return linear_fwd_bf16(*desc, p, x, W, bias, residual, drop, rng_used, y, saved, ws, (hipStream_t)hip_stream);
    return linear_fwd_f32(*desc, p, (const float*)x, (const float*)W, bias, (const float*)residual, drop, rng_used, (float*)y, (float*)saved, ws,
                          (hipStream_t)hip_stream);
}

extern "C" rnnt_status rnnt_linear_bwd(const rnnt_linear_desc* desc, const void* x, const void* W, const void* saved, const uint64_t* rng,
                                       const void* dy, void* dx, void* dW, void* db, void* workspace, size_t workspace_bytes, void* hip_stream) {
    const rnnt_status st = check_linear(desc, true);
    if (st != RNNT_OK) return st;
    if (!W || (desc->M > 0 && (!x || !dy || (desc->activation != ACT_NONE && !saved)))) return RNNT_ERR_NULL;
    const Dropout drop = make_dropout(*desc, rng);
    if (drop.cut != 0 && !rng) return RNNT_ERR_NULL;
    if (!aligned({x, W, saved, dy, dx, dW, db}) || (uintptr_t)rng % 8 != 0) return RNNT_ERR_UNSUPPORTED;
    const LinearPlan p = plan_linear(*desc, true);
    if (!workspace_ok(workspace, workspace_bytes, p.bytes)) return RNNT_ERR_WORKSPACE;
    unsigned char* ws = (unsigned char*)workspace;
    if (p.bf16) return linear_bwd_bf16(*desc, p, x, W, saved, drop, dy, dx, dW, db, ws, (hipStream_t)hip_stream);
    return linear_bwd_f32(*desc, p, (const float*)x, (const float*)W, (const float*)saved, drop, (const float*)dy, (float*)dx, (float*)dW, (float*)db, ws,
                          (hipStream_t)hip_stream);
}

extern "C" size_t rnnt_ce_loss_workspace_bytes(const rnnt_ce_desc* desc, int32_t grads, size_t budget_bytes) {
    if (check_ce(desc, grads != 0) != RNNT_OK) return 0;
    return plan_ce(*desc, grads != 0, budget_bytes).bytes;
}

static rnnt_status ce_loss(const rnnt_ce_desc* desc, bool grads, const void* x, const void* W, const void* b, const int32_t* label,
                           const float* row_weight, float* loss, void* dx, void* dW, void* db, void* workspace, size_t workspace_bytes,
                           void* hip_stream) {
    const rnnt_status st = check_ce(desc, grads);
    if (st != RNNT_OK) return st;
    if (!W || (grads && !dW) || (desc->R > 0 && (!x || !label || !loss || (grads && !dx)))) return RNNT_ERR_NULL;
    if (!aligned({x, W, b, dx, dW, db}) || (((uintptr_t)label | (uintptr_t)row_weight | (uintptr_t)loss) % 4) != 0) return RNNT_ERR_UNSUPPORTED;
    // the default plan where it fits, larger chunks in a larger workspace, smaller ones in a smaller
    CePlan p = plan_ce(*desc, grads, 0);
    if (workspace_bytes != p.bytes && (p.chunks > 1 || workspace_bytes < p.bytes)) {
        const CePlan q = plan_ce(*desc, grads, workspace_bytes == 0 ? 1 : workspace_bytes);
        if (workspace_bytes < p.bytes || q.chunk > p.chunk) p = q;
    }
    if (!workspace_ok(workspace, workspace_bytes, p.bytes)) return RNNT_ERR_WORKSPACE;
    return run_ce(*desc, p, x, W, b, label, row_weight, loss, dx, dW, db, (unsigned char*)workspace, (hipStream_t)hip_stream);
}

extern "C" rnnt_status rnnt_ce_loss_fwd(const rnnt_ce_desc* desc, const void* x, const void* W, const void* b, const int32_t* label, float* loss,
                                        void* workspace, size_t workspace_bytes, void* hip_stream) {
    return ce_loss(desc, false, x, W, b, label, nullptr, loss, nullptr, nullptr, nullptr, workspace, workspace_bytes, hip_stream);
}
extern "C" rnnt_status rnnt_ce_loss_fwd_bwd(const rnnt_ce_desc* desc, const void* x, const void* W, const void* b, const int32_t* label,
                                            const float* row_weight, float* loss, void* dx, void* dW, void* db, void* workspace,
                                            size_t workspace_bytes, void* hip_stream) {
    return ce_loss(desc, true, x, W, b, label, row_weight, loss, dx, dW, db, workspace, workspace_bytes, hip_stream);
}
extern "C" rnnt_status rnnt_ce_loss_total(const rnnt_ce_desc* desc, const float* loss, const float* row_weight, float* total, void* hip_stream) {
    const rnnt_status st = check_ce(desc, false);
    if (st != RNNT_OK) return st;
    if (!total || (desc->R > 0 && !loss)) return RNNT_ERR_NULL;
    if ((((uintptr_t)loss | (uintptr_t)row_weight | (uintptr_t)total) % 4) != 0) return RNNT_ERR_UNSUPPORTED;
    LAYER_HIP(launch_ce_total(loss, row_weight, desc->R, total, (hipStream_t)hip_stream));
    return RNNT_OK;
}
extern "C" rnnt_status rnnt_ce_loss_scale(const rnnt_ce_desc* desc, const float* factor, void* dx, void* dW, void* db, void* hip_stream) {
    const rnnt_status st = check_ce(desc, true);
    if (st != RNNT_OK) return st;
    if (!factor) return RNNT_ERR_NULL;
    if (!aligned({dx, dW, db}) || (uintptr_t)factor % 4 != 0) return RNNT_ERR_UNSUPPORTED;
    const long long n[3] = {dx ? desc->R * desc->D : 0, dW ? (long long)desc->D * desc->V : 0, db ? desc->V : 0};
    const bool bf16[3] = {desc->dtype == RNNT_BF16, (desc->param_grads_bf16 & 1) != 0, (desc->param_grads_bf16 & 2) != 0};
    void* const p[3] = {dx, dW, db};
    LAYER_HIP(launch_scale(factor, p, n, bf16, (hipStream_t)hip_stream));
    return RNNT_OK;
}
