// Element-wise mathematics of the linear layer and its epilogues (device code).
#pragma once
#include "device_common.h"
#include "layers.h"

namespace rnnt {

namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers, as easy as 1, 2, 3; 2011) with key {seed} on the counter {column / 8, row, offset}:
// the 128 bits of eight columns, 16 for each.
struct RandomBits8 {
    unsigned w[4];
    __device__ __forceinline__ unsigned of(int j) const { return (j & 1) ? w[j >> 1] >> 16 : w[j >> 1] & 0xffffu; }
};
__device__ __forceinline__ RandomBits8 random_bits8(unsigned long long seed, unsigned long long offset, unsigned row, unsigned group) {
    unsigned c0 = group, c1 = row, c2 = (unsigned)offset, c3 = (unsigned)(offset >> 32), k0 = (unsigned)seed, k1 = (unsigned)(seed >> 32);
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const unsigned h0 = __umulhi(c0, 0xD2511F53u), l0 = c0 * 0xD2511F53u, h1 = __umulhi(c2, 0xCD9E8D57u), l1 = c2 * 0xCD9E8D57u;
        c0 = h1 ^ c1 ^ k0;
        c1 = l1;
        c2 = h0 ^ c3 ^ k1;
        c3 = l0;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return RandomBits8{{c0, c1, c2, c3}};
}
// v[j] *= mask / (1 - p), columns n .. n + 7 of row m (n a multiple of 8).  A dropped entry is 0 whatever it was.
__device__ __forceinline__ void drop8(const Dropout& d, long long m, int n, float (&v)[8]) {
    if (d.cut == 0) return;
    const RandomBits8 r = random_bits8(d.state[0], d.state[1], (unsigned)m, (unsigned)n >> 3);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = r.of(j) >= d.cut ? v[j] * d.scale : 0.0f;
}

// FAST: by the exponential and reciprocal instructions (relative error about 1e-6, results that are rounded to bf16); else the math library's functions.
template <bool FAST>
__device__ __forceinline__ float sigmoid(float x) {
    if constexpr (FAST) return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-LOG2E_F * x));
    else return 1.0f / (1.0f + expf(-x));
}
template <bool FAST>
__device__ __forceinline__ void act8(int act, float (&v)[8]) {
    switch (act) {
        case ACT_RELU:
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = v[j] < 0.0f ? 0.0f : v[j];          // (keeps NaN)
            break;
        case ACT_SILU:
            // (-inf: 0, the limit)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = v[j] == RNNT_NEG_INF ? 0.0f : v[j] * sigmoid<FAST>(v[j]);
            break;
        case ACT_GELU:
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = v[j] == RNNT_NEG_INF ? 0.0f : v[j] * (0.5f * erfcf(-0.70710678118654752f * v[j]));
            break;
        case ACT_TANH:
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = FAST ? fast_tanh(v[j]) : tanhf(v[j]);
            break;
        default: break;
    }
}
// g[j] *= act'(z[j]); z finite or NaN
template <bool FAST>
__device__ __forceinline__ void act_grad8(int act, const float (&z)[8], float (&g)[8]) {
    switch (act) {
        case ACT_RELU:
#pragma unroll
            for (int j = 0; j < 8; ++j) g[j] = z[j] > 0.0f ? g[j] : z[j] <= 0.0f ? 0.0f : z[j];
            break;
        case ACT_SILU:
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float p = sigmoid<FAST>(z[j]), q = sigmoid<FAST>(-z[j]);     // (1 - p would lose it where p is near 1)
                g[j] *= p * fmaf(z[j], q, 1.0f);
            }
            break;
        case ACT_GELU:
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float x = z[j], d = FAST ? __builtin_amdgcn_exp2f(-0.5f * LOG2E_F * x * x) : expf(-0.5f * x * x);
                g[j] *= fmaf(x * 0.3989422804014327f, d, 0.5f * erfcf(-0.70710678118654752f * x));
            }
            break;
        case ACT_TANH:
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                // 1 - tanh^2 = 4 p q with p, q = sigmoid(+-2z)
                g[j] *= 4.0f * sigmoid<FAST>(2.0f * z[j]) * sigmoid<FAST>(-2.0f * z[j]);
            }
            break;
        default: break;
    }
}

// A saved pre-activation: fp16 (11 bits, where bf16's eight would add as much to the gradient's error as its own rounding does), beyond the largest
// one that largest one (there act' has its limit), and a nonzero one stays nonzero (its sign is relu's derivative).
__device__ __forceinline__ _Float16 saved_f16(float z) {
    float c = z > 65504.0f ? 65504.0f : z < -65504.0f ? -65504.0f : z;             // (NaN stays)
    if (c > 0.0f && c < 5.9604644775390625e-8f) c = 5.9604644775390625e-8f;
    if (c < 0.0f && c > -5.9604644775390625e-8f) c = -5.9604644775390625e-8f;
    return (_Float16)c;
}

// ---- what becomes of columns n .. n + 7 (n a multiple of 8) of row m of a product --------------------------------------
__device__ __forceinline__ void load_bias8(const float* bias, int n, int N, float (&b)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) b[j] = bias != nullptr ? bias[n + j < N ? n + j : N - 1] : 0.0f;
}
struct LinearStore {
    __device__ static __forceinline__ void store(const LinearEpilogue& e, int, long long m, int n, float (&v)[8], const float (&b)[8]) {
        if (m >= e.M || n >= e.N) return;
        const size_t at = (size_t)m * e.N + n;
        const int live = e.N - n < 8 ? e.N - n : 8;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += b[j];
        if (e.saved != nullptr) {
            _Float16* s = (_Float16*)e.saved + at;
            f16x8 h;
#pragma unroll
            for (int j = 0; j < 8; ++j) h[j] = saved_f16(v[j]);
            if (e.vec) *reinterpret_cast<f16x8*>(s) = h;
            else
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < live) s[j] = h[j];
        }
        act8<true>(e.act, v);
        drop8(e.drop, m, n, v);
        if (e.residual != nullptr) {
            const bf16_t* r = (const bf16_t*)e.residual + at;
            if (e.vec) {
                const bf16x8 x = *reinterpret_cast<const bf16x8*>(r);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] += (float)x[j];
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] += (float)r[j < live ? j : 0];
            }
        }
        bf16_t* y = (bf16_t*)e.y + at;
        if (e.vec) {
            bf16x8 o;
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = (bf16_t)v[j];
            *reinterpret_cast<bf16x8*>(y) = o;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < live) y[j] = (bf16_t)v[j];
        }
    }
    __device__ static __forceinline__ void bias(const LinearEpilogue& e, int n, float (&b)[8]) { load_bias8(e.bias, n < e.N ? n : e.N - 1, e.N, b); }
};
struct PlainStore {
    __device__ static __forceinline__ void store(const StoreEpilogue& e, int split, long long m, int n, float (&v)[8], const float (&)[8]) {
        if (m >= e.M || n >= e.N) return;
        long long row = m;
        if (e.row_map != nullptr) {
            row = e.row_map[m];
            if (row < 0) return;
        }
        const size_t at = (size_t)split * e.split_stride + (size_t)row * e.ld + n;
        const int live = e.N - n < 8 ? e.N - n : 8;
        if (e.prev != nullptr) {
            if (e.vec) {
                const f32x4 a = *reinterpret_cast<const f32x4*>(e.prev + at), b = *reinterpret_cast<const f32x4*>(e.prev + at + 4);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    v[j] += a[j];
                    v[4 + j] += b[j];
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] += e.prev[at + (j < live ? j : 0)];
            }
        }
        if (e.bf16) {
            bf16_t* o = (bf16_t*)e.out + at;
            bf16x8 x;
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = (bf16_t)v[j];
            if (e.vec) *reinterpret_cast<bf16x8*>(o) = x;
            else
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < live) o[j] = x[j];
        } else {
            float* o = (float*)e.out + at;
            if (e.vec) {
                *reinterpret_cast<f32x4*>(o) = f32x4{v[0], v[1], v[2], v[3]};
                *reinterpret_cast<f32x4*>(o + 4) = f32x4{v[4], v[5], v[6], v[7]};
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < live) o[j] = v[j];
            }
        }
    }
    __device__ static __forceinline__ void bias(const StoreEpilogue&, int, float (&b)[8]) {
#pragma unroll
        for (int j = 0; j < 8; ++j) b[j] = 0.0f;
    }
};
template <class E>
struct EpilogueOf;
template <>
struct EpilogueOf<LinearEpilogue> {
    typedef LinearStore type;
};
template <>
struct EpilogueOf<StoreEpilogue> {
    typedef PlainStore type;
};

}  // namespace

}  // namespace rnnt
