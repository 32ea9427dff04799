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

// Where the operands of the products lie.  bf16: as the caller has them where rows are multiples of 64 elements along a contiguous contraction and of 8 along the
// other index, else in a padded copy.  fp32: in a padded copy as parts (layers.h).
struct LinearPlan {
    bool f32, few;                        // few: forward pass of at most FEW_ROWS rows, one launch on the arrays as they are
    int few_splits;
    bool copy_x, copy_w, own_dz;
    bool rest;                            // backward: dz in two bf16 values, the rounded one and the rest
    long long Kp, Np, Mp;                 // multiples of 64
    size_t off_x, off_w, off_dz, off_xt, off_dyt, off_part, off_slots, off_slots_w, bytes;
    GemmPlan y;
    PairPlan grads;
};
LinearPlan plan_linear(const rnnt_linear_desc& d, bool backward) {
    LinearPlan p{};
    p.f32 = d.dtype == RNNT_F32;
    const long long M = d.M, K = d.K, N = d.N;
    const int per = p.f32 ? PAIRS : 1;    // stages per 64 of depth
    const size_t e = p.f32 ? PARTS * 2 : 2;
    const bool plain = d.activation == ACT_NONE && dropout_cut(d.dropout) == 0;
    Carver c;
    p.Kp = up(K, 64);
    p.Np = up(N, 64);
    p.Mp = up(M, 64);
    if (!backward && M <= FEW_ROWS) {
        p.few = true;
        p.few_splits = few_splits(p.f32, M, d.K, d.N);
        p.off_slots = c.take(p.few_splits > 1 ? (size_t)p.few_splits * M * up(N, 8) * 4 : 0);
    } else if (!backward) {
        p.copy_x = p.f32 || K % 64 != 0;
        p.copy_w = p.f32 || K % 64 != 0 || N % 8 != 0;
        p.y = plan_gemm(M, N, (int)(p.Kp / 64) * per, SLOT_CAP);
        p.off_x = c.take(p.copy_x ? (size_t)M * p.Kp * e : 0);
        p.off_w = c.take(p.copy_w ? (size_t)p.Kp * p.Np * e : 0);
        p.off_slots = c.take(gemm_slot_bytes(p.y, M, N));
    } else {
        p.own_dz = p.f32 || !plain || N % 64 != 0;
        p.copy_x = p.f32 || K % 8 != 0;
        p.copy_w = p.f32 || N % 64 != 0;
        p.rest = !p.f32 && M <= FEW_ROWS && d.activation != ACT_NONE && d.activation != ACT_RELU;
        const int passes = p.rest ? 2 : per;
        p.grads = plan_pair(M, K, (int)(p.Np / 64) * passes, K, N, (int)(p.Mp / 64) * passes, SLOT_CAP, p.rest);
        p.off_dz = c.take(p.own_dz ? (size_t)p.Mp * p.Np * e * (p.rest ? 2 : 1) : 0);
        p.off_x = c.take(p.copy_x ? (size_t)p.Mp * p.Kp * e : 0);
        p.off_w = c.take(p.copy_w ? (size_t)K * p.Np * e : 0);
        p.off_xt = c.take(!p.copy_x && M % 64 != 0 ? (size_t)64 * K * 2 : 0);
        p.off_dyt = c.take(!p.own_dz && M % 64 != 0 ? (size_t)64 * N * 2 : 0);
        p.off_part = c.take((size_t)sum_capacity(M, N) * p.Np * 4);
        p.off_slots = c.take(gemm_slot_bytes(p.grads.dx, M, K));
        p.off_slots_w = c.take(gemm_slot_bytes(p.grads.dw, K, N));
    }
    p.bytes = c.bytes;
    return p;
}

// An operand: the caller's array of pitch ld, or a copy of `rows` rows of pitch ld_copy
GemmOperand operand(bool copied, bool f32, const void* own, long long ld, const void* copy, long long rows, long long ld_copy) {
    return copied ? GemmOperand{copy, ld_copy, f32 ? rows * ld_copy : 0, nullptr, -1, 0} : GemmOperand{own, ld, 0, nullptr, -1, 0};
}

// A bf16 product with an operand in two values: `once` by the rounded ones, then by the rest.
// Rounding the gradient to bf16 adds as much to the products' error as their own rounding does, sqrt(2) times it where many values average; the few of a few
// rows do not (up to 3 times).  There, up to FEW_ROWS rows, the products wait for W and dW rather than for their operations (backward pass of 64 x 512 x 2048
// in a captured graph 14.5 us with dz in one value (relu), 17.2 in two (silu); 64 x 1024 x 4096 20.4 and 23.3).
void take_twice(GemmOperand& once, GemmOperand& two, long long rest, int stages) {
    once.wrap = two.wrap = stages;
    two.part = rest;
}

rnnt_status linear_fwd(const rnnt_linear_desc& d, const LinearPlan& p, const void* x, const void* W, const Bias& b, const void* residual,
                       const Dropout& drop, uint64_t* rng_used, void* y, void* saved, unsigned char* ws, hipStream_t stream) {
    const long long M = d.M, K = d.K, N = d.N;
    const LinearEpilogue e{b, residual, y, saved, d.activation, drop, (unsigned long long*)rng_used, M, d.N};
    float* slots = (float*)(ws + p.off_slots);
    if (p.few) {
        LAYER_HIP(launch_few_linear(FewJob{x, W, (int)M, d.K, d.N, p.f32}, p.few_splits, slots, e, stream));
        return RNNT_OK;
    }
    const int kind = p.f32 ? PAD_PARTS : PAD_16;
    PadJobs pads{};
    if (p.copy_x) pads.add(kind, x, M, K, 0, ws + p.off_x, M, p.Kp);
    if (p.copy_w) pads.add(kind, W, K, N, 0, ws + p.off_w, p.Kp, p.Np);
    LAYER_HIP(launch_pads(pads, stream));
    GemmJob g{};
    g.A = operand(p.copy_x, p.f32, x, K, ws + p.off_x, M, p.Kp);
    g.B = operand(p.copy_w, p.f32, W, N, ws + p.off_w, p.Kp, p.Np);
    g.M = g.a_rows = M;
    g.N = N;
    g.b_rows = p.copy_w ? p.Np : N;
    g.per_block = p.f32 ? PAIRS : 1;
    g.stages = (int)(p.Kp / 64) * g.per_block;
    LAYER_HIP(p.f32 ? launch_linear_gemm(g, p.y, slots, LinearEpilogue32{e}, stream) : launch_linear_gemm(g, p.y, slots, e, stream));
    return RNNT_OK;
}

rnnt_status linear_bwd(const rnnt_linear_desc& d, const LinearPlan& p, const void* x, const void* W, const void* saved, const Dropout& drop, const void* dy,
                       void* dx, void* dW, void* db, unsigned char* ws, hipStream_t stream) {
    const long long M = d.M, K = d.K, N = d.N, whole = M / 64 * 64;
    const bool ragged = M % 64 != 0;
    float* part = (float*)(ws + p.off_part);
    Dropout mask = drop;                  // (its factor: in the products' epilogues)
    mask.scale = 1.0f;
    const long long rest = p.rest ? p.Mp * p.Np : 0;
    if (M == 0) dx = nullptr;
    const int kind = p.f32 ? PAD_PARTS : PAD_16;
    PadJobs pads{};
    if (dx && p.copy_w) pads.add(kind, W, K, N, 0, ws + p.off_w, K, p.Np);
    if (dW && p.copy_x) pads.add(kind, x, M, K, 0, ws + p.off_x, p.Mp, p.Kp);
    else if (dW && ragged) pads.add(PAD_16, x, M, K, whole, ws + p.off_xt, 64, K);
    if (dW && !p.own_dz && ragged) pads.add(PAD_16, dy, M, N, whole, ws + p.off_dyt, 64, N);
    if (M > 0 && (db || (p.own_dz && (dx || dW)))) {
        const DzArgs a{dy, d.activation == ACT_NONE ? nullptr : saved, p.own_dz && (dx || dW) ? ws + p.off_dz : nullptr, db ? part : nullptr, M,
                       p.own_dz ? p.Mp : M, d.N, p.Np, d.activation, mask, rest};
        LAYER_HIP(launch_dz(!p.f32, a, pads, stream));
    } else LAYER_HIP(launch_pads(pads, stream));
    GradGemm gx{}, gw{};
    gx.g.per_block = gw.g.per_block = p.f32 ? PAIRS : p.rest ? 2 : 1;
    const GemmOperand dz = operand(p.own_dz, p.f32, dy, N, ws + p.off_dz, p.Mp, p.Np);
    if (dx) {
        gx.g.A = dz;
        gx.g.B = operand(p.copy_w, p.f32, W, N, ws + p.off_w, K, p.Np);
        gx.g.M = gx.g.a_rows = M;
        gx.g.N = gx.g.b_rows = K;
        gx.g.stages = (int)(p.Np / 64) * gx.g.per_block;
        gx.splits = p.grads.dx.splits;
        gx.per_split = p.grads.dx.per_split;
        gx.slots = (float*)(ws + p.off_slots);
        if (p.rest) take_twice(gx.g.B, gx.g.A, rest, (int)(p.Np / 64));
        gx.e = StoreEpilogue{dx, nullptr, drop.scale, nullptr, nullptr, K, 0, Bias{}, M, d.K, !p.f32};
    }
    if (dW) {
        gw.g.A = operand(p.copy_x, p.f32, x, K, ws + p.off_x, p.Mp, p.Kp);
        gw.g.B = dz;
        if (ragged && !p.copy_x) gw.g.A.tail = ws + p.off_xt;
        if (ragged && !p.own_dz) gw.g.B.tail = ws + p.off_dyt;
        gw.g.A.tail_stage = gw.g.B.tail_stage = (int)(whole / 64);
        gw.g.M = K;
        gw.g.a_rows = p.copy_x ? p.Kp : K;
        gw.g.N = N;
        gw.g.b_rows = p.own_dz ? p.Np : N;
        gw.g.stages = (int)(p.Mp / 64) * gw.g.per_block;
        gw.splits = p.grads.dw.splits;
        gw.per_split = p.grads.dw.per_split;
        gw.slots = (float*)(ws + p.off_slots_w);
        if (p.rest) take_twice(gw.g.A, gw.g.B, rest, (int)(p.Mp / 64));
        gw.e = StoreEpilogue{dW, d.accumulate_params ? (const float*)dW : nullptr, drop.scale, nullptr, nullptr, N, 0, Bias{}, K, d.N, (d.param_grads_bf16 & 1) != 0};
    }
    // (whether it is wanted is told by db: without rows the workspace, and with it `part`, may be null)
    const SumJob sum{part, M, p.Np, d.N, nullptr, 0, d.accumulate_params ? (const float*)db : nullptr, db, (d.param_grads_bf16 & 2) != 0, drop.scale, nullptr};
    LAYER_HIP(launch_grad_gemms(p.f32, p.grads.tile, gx, gw, sum, stream));
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
    bool f32, grads, copy_w;
    bool few;                             // at most FEW_ROWS rows (fp32: without gradients): scores by one launch on W as it is
    bool identity;                        // ... and without gradients on x as it is
    long long rest;                       // elements from a chunk's score gradients to their rests (few; 0: none)
    long long cap, chunk, Dp, Vp, pitch;  // rows (a multiple of 256) in all and per chunk; widths up to 64; elements of a chunk row
    int chunks, tile, tile_log2, tiles_n;
    size_t off_count, off_index, off_label, off_weight, off_place, off_x, off_w, off_chunk, off_grad, off_score, off_stats, off_scale, off_part, off_slots,
        off_slots_w, off_acc, off_dbacc, bytes;
    PairPlan pair;
};
CePlan plan_ce_chunk(const rnnt_ce_desc& d, bool grads, long long chunk) {
    CePlan p{};
    p.f32 = d.dtype == RNNT_F32;
    p.grads = grads;
    const long long R = d.R, D = d.D, V = d.V;
    const int per = p.f32 ? PAIRS : 1;
    const size_t e = p.f32 ? PARTS * 2 : 2;
    p.cap = std::max(256LL, up(R, 256));
    p.chunk = std::min(chunk, p.cap);
    p.chunks = (int)((p.cap + p.chunk - 1) / p.chunk);
    p.Dp = up(D, 64);
    p.Vp = up(V, 64);
    p.few = R <= FEW_ROWS && !(p.f32 && grads);
    p.identity = p.few && !grads;
    p.copy_w = !p.identity && (p.f32 || p.Dp != D || p.Vp != V);
    p.tile = p.few ? FEW_TILE : plan_gemm(p.chunk, V, (int)(p.Dp / 64) * per, 0).tile;
    p.tile_log2 = p.few ? 5 : p.tile == 256 ? 8 : 7;
    // (few, on a copy of W: the columns of zeros up to Vp have parts of their own)
    p.tiles_n = (int)(((p.few && !p.identity ? p.Vp : V) + p.tile - 1) / p.tile);
    Carver c;
    if (p.identity) {
        p.off_score = c.take((size_t)FEW_ROWS * 4);
        p.off_stats = c.take((size_t)R * p.tiles_n * 8);
        p.bytes = c.bytes;
        return p;
    }
    p.off_count = c.take(4);
    p.off_index = c.take((size_t)p.cap * 4);
    p.off_label = c.take((size_t)p.cap * 4);
    p.off_weight = c.take((size_t)p.cap * 4);
    p.off_place = c.take(R > GATHER_SCAN ? (size_t)ce_place_ints(p.cap) * 4 : 0);
    p.off_x = c.take((size_t)p.cap * p.Dp * e);
    p.off_w = c.take(p.copy_w ? (size_t)p.Dp * p.Vp * e : 0);
    if (p.f32) {
        p.pitch = p.Vp;
        p.off_chunk = c.take((size_t)p.chunk * p.pitch * 4);
        p.off_grad = c.take(grads ? (size_t)p.chunk * p.pitch * e : 0);
    } else {
        // (a row is 128 bytes longer than whole tiles: rows of a power-of-two length would all start in the same memory channel)
        p.pitch = up(V, 256) + 64;
        p.off_score = c.take((size_t)p.chunk * 4);
        p.off_stats = c.take((size_t)p.chunk * p.tiles_n * 8);
        p.off_scale = c.take((size_t)p.chunk * 16);
        p.rest = grads && p.few ? p.chunk * p.pitch : 0;
        p.off_chunk = p.off_grad = c.take(grads ? (size_t)(p.chunk * p.pitch + p.rest) * 2 : 0);
    }
    if (grads) {
        p.off_part = c.take((size_t)sum_capacity(p.chunk, V) * p.pitch * 4);
        // (few: 64 rows, twice)
        p.pair = p.rest ? plan_pair(FEW_ROWS, D, (int)(p.Vp / 64) * 2, D, V, 2, SLOT_CAP, true)
                        : plan_pair(p.chunk, D, (int)(p.Vp / 64) * per, D, V, (int)(p.chunk / 64) * per, SLOT_CAP, false);
        p.off_slots = c.take(gemm_slot_bytes(p.pair.dx, p.chunk, D));
        p.off_slots_w = c.take(gemm_slot_bytes(p.pair.dw, D, V));
        // the weight gradient's sum over the chunks, where its output is bfloat16
        p.off_acc = c.take(p.chunks > 1 && (d.param_grads_bf16 & 1) ? (size_t)D * V * 4 : 0);
        p.off_dbacc = c.take(p.chunks > 1 ? (size_t)V * 4 : 0);
    }
    p.bytes = c.bytes;
    return p;
}
// Equal chunks, as few as a plan of at most `budget` bytes has (0: as chunk buffers of at most CE_CHUNK allow); the plan of fewest bytes where none does.
// A plan's bytes do not grow with its chunks: a single one needs no sums over the chunks (D x V floats), and longer ones take fewer splits.  So every number of
// chunks that can fit is looked at (1 us each).  The plan for a budget of its own bytes is itself.
CePlan plan_ce(const rnnt_ce_desc& d, bool grads, size_t budget) {
    const bool f32 = d.dtype == RNNT_F32;
    const long long all = std::max(256LL, up(d.R, 256));
    const size_t row = f32 ? (size_t)up(d.V, 64) * (4 + (grads ? PARTS * 2 : 0)) : (size_t)(up(d.V, 256) + 64) * 2;
    // the chunks where each takes at most `rows` rows, a multiple of 256
    auto equal = [&](long long rows) {
        const long long n = (all + rows - 1) / rows;
        return up((all + n - 1) / n, 256);
    };
    if (budget == 0) return plan_ce_chunk(d, grads, equal(std::max(256LL, (long long)(CE_CHUNK / row) / 256 * 256)));
    // (losses alone of RNNT_BF16 keep no exponentials)
    const size_t most = f32 || grads ? budget / row : (size_t)all;
    for (long long c = equal(std::max(256LL, (long long)std::min(most, (size_t)all) / 256 * 256));; c = equal(c - 256)) {
        const CePlan p = plan_ce_chunk(d, grads, c);
        if (p.bytes <= budget) return p;
        if (c <= 256) break;
    }
    CePlan least = plan_ce_chunk(d, grads, all);
    for (long long c = all; c > 256;) {
        c = equal(c - 256);
        const CePlan p = plan_ce_chunk(d, grads, c);
        if (p.bytes < least.bytes) least = p;
    }
    return least;
}

rnnt_status run_ce(const rnnt_ce_desc& d, const CePlan& p, const void* x, const void* W, const Bias& b, const int32_t* label, const float* row_weight,
                   float* loss, void* dx, void* dW, void* db, unsigned char* ws, hipStream_t stream) {
    const long long D = d.D, V = d.V;
    if (!p.grads && d.R == 0) return RNNT_OK;
    if (p.identity) {
        CeRows own{};
        own.label = const_cast<int*>(label);
        const CeEpilogue e{b, d.V, label, (float*)(ws + p.off_score), (float2*)(ws + p.off_stats), p.tiles_n, nullptr, 0};
        LAYER_HIP(launch_few_ce(FewJob{x, W, (int)d.R, d.D, d.V, p.f32}, e, stream));
        LAYER_HIP(launch_ce_finish(CeChunk{own, 0, d.R, e.label_score, e.stats, p.tiles_n, p.tile_log2, d.V, nullptr, loss, true, d.ignore_label}, stream));
        return RNNT_OK;
    }
    const CeRows rows{(int*)(ws + p.off_count), (int*)(ws + p.off_index), (int*)(ws + p.off_label), (float*)(ws + p.off_weight)};
    const int kind = p.f32 ? PAD_PARTS : PAD_16;
    PadJobs pads{};
    if (d.R == 0) pads.add(PAD_32, nullptr, 0, 0, 0, rows.count, 1, 8);       // (the gradients of an empty sum; the part behind is 256 bytes away)
    if (p.copy_w) pads.add(kind, W, D, V, 0, ws + p.off_w, p.Dp, p.Vp);
    if (d.R > 0)
        LAYER_HIP(launch_ce_gather(x, p.f32, d.R, d.D, label, row_weight, d.ignore_label, p.cap, (int*)(ws + p.off_place), rows, ws + p.off_x, p.Dp, loss,
                                   p.grads ? dx : nullptr, pads, stream));
    else LAYER_HIP(launch_pads(pads, stream));
    const GemmOperand w = operand(p.copy_w, p.f32, W, V, ws + p.off_w, p.Dp, p.Vp);
    unsigned char *chunk = ws + p.off_chunk, *grad = ws + p.off_grad;
    float* part = (float*)(ws + p.off_part);
    for (int k = 0; k < p.chunks; ++k) {
        const long long row0 = (long long)k * p.chunk, n = p.rest ? FEW_ROWS : std::min(p.chunk, p.cap - row0);
        const bool first = k == 0, last = k == p.chunks - 1;
        GemmJob g{};
        g.A = GemmOperand{ws + p.off_x + (size_t)row0 * p.Dp * 2, p.Dp, p.f32 ? p.cap * p.Dp : 0, nullptr, -1, 0};
        g.B = w;
        g.M = g.a_rows = n;
        g.N = V;
        g.b_rows = p.Vp;
        g.per_block = p.f32 ? PAIRS : 1;
        g.stages = (int)(p.Dp / 64) * g.per_block;
        g.limit = GEMM_ROWS_M;
        g.count = rows.count;
        g.row0 = row0;
        if (d.R == 0) {
        } else if (p.f32) {
            const StoreEpilogue e{chunk, nullptr, 1.0f, nullptr, nullptr, p.pitch, 0, b, n, d.V, false};
            LAYER_HIP(launch_scores_f32(g, p.tile, e, stream));
            LAYER_HIP(launch_ce_rows_f32(rows, row0, n, (const float*)chunk, p.pitch, d.V, loss, p.grads ? grad : nullptr, stream));
            if (p.grads && db) LAYER_HIP(launch_col_sums_f32(grad, n, p.pitch, d.V, rows.count, row0, part, stream));
        } else {
            const CeEpilogue e{b, d.V, rows.label + row0, (float*)(ws + p.off_score), (float2*)(ws + p.off_stats), p.tiles_n,
                               p.grads ? chunk : nullptr, p.pitch};
            const CeChunk c{rows, row0, n, e.label_score, e.stats, p.tiles_n, p.tile_log2, d.V, (float4*)(ws + p.off_scale), loss, false, 0};
            if (p.few) LAYER_HIP(launch_few_ce(FewJob{g.A.p, w.p, (int)d.R, (int)p.Dp, (int)p.Vp, false}, e, stream));
            else LAYER_HIP(launch_ce_gemm(g, p.tile, e, stream));
            if (!p.grads || !ce_grad_finishes(n, V, p.tiles_n)) LAYER_HIP(launch_ce_finish(c, stream));
            if (p.grads) LAYER_HIP(launch_ce_grad(c, chunk, p.pitch, p.rest, db ? part : nullptr, stream));
        }
        if (!p.grads) continue;
        const GemmOperand dh{grad, p.pitch, p.f32 ? n * p.pitch : 0, nullptr, -1, 0};
        const float* unit = p.f32 ? nullptr : ce_unit(rows);
        GradGemm gx{}, gw{};
        const int per = p.rest ? 2 : g.per_block;
        if (d.R > 0) {
            gx.g = g;
            gx.g.A = dh;
            gx.g.N = gx.g.b_rows = D;
            gx.g.per_block = per;
            gx.g.stages = (int)(p.Vp / 64) * per;
            if (p.rest) take_twice(gx.g.B, gx.g.A, p.rest, (int)(p.Vp / 64));
            gx.splits = p.pair.dx.splits;
            gx.per_split = p.pair.dx.per_split;
            gx.slots = (float*)(ws + p.off_slots);
            gx.e = StoreEpilogue{dx, nullptr, 1.0f, unit, rows.index + row0, D, 0, Bias{}, n, d.D, !p.f32};
        }
        gw.g.A = g.A;
        gw.g.B = dh;
        gw.g.M = D;
        gw.g.a_rows = p.Dp;
        gw.g.N = V;
        gw.g.b_rows = p.Vp;
        gw.g.per_block = per;
        gw.g.stages = (int)(n / 64) * per;
        if (p.rest) take_twice(gw.g.A, gw.g.B, p.rest, 1);
        gw.g.limit = GEMM_ROWS_K;
        gw.g.count = rows.count;
        gw.g.row0 = row0;
        gw.splits = p.pair.dw.splits;
        gw.per_split = p.pair.dw.per_split;
        gw.slots = (float*)(ws + p.off_slots_w);
        const bool w16 = (d.param_grads_bf16 & 1) != 0, b16 = (d.param_grads_bf16 & 2) != 0;
        float* acc = w16 ? (float*)(ws + p.off_acc) : (float*)dW;
        gw.e = StoreEpilogue{last ? dW : acc, !first || d.accumulate_params ? acc : nullptr, 1.0f, unit, nullptr, V, 0, Bias{}, D, d.V, last && w16};
        float* dba = (float*)(ws + p.off_dbacc);
        const SumJob sum{part, n, p.pitch, d.V, rows.count, row0, first ? (d.accumulate_params ? (const float*)db : nullptr) : dba,
                         last || !db ? db : (void*)dba, last && b16, 1.0f, unit};
        LAYER_HIP(launch_grad_gemms(p.f32, p.pair.tile, gx, gw, sum, stream));
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
    if (desc->M == 0) {
        if (rng_used) LAYER_HIP(launch_pass_rng(drop.state, (unsigned long long*)rng_used, (hipStream_t)hip_stream));
        return RNNT_OK;
    }
    unsigned char* ws = (unsigned char*)workspace;
    const Bias bias{b, desc->bias_bf16 != 0};
    return linear_fwd(*desc, p, x, W, bias, residual, drop, rng_used, y, saved, ws, (hipStream_t)hip_stream);
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
    return linear_bwd(*desc, p, x, W, saved, drop, dy, dx, dW, db, ws, (hipStream_t)hip_stream);
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
    if (workspace_bytes < p.bytes || (workspace_bytes > p.bytes && p.chunks > 1)) p = plan_ce(*desc, grads, workspace_bytes == 0 ? 1 : workspace_bytes);
    if (!workspace_ok(workspace, workspace_bytes, p.bytes)) return RNNT_ERR_WORKSPACE;
    return run_ce(*desc, p, x, W, Bias{b, desc->bias_bf16 != 0}, label, row_weight, loss, dx, dW, db, (unsigned char*)workspace, (hipStream_t)hip_stream);
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
