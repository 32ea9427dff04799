// Element-wise mathematics of the linear layer and its epilogues (device code).
#pragma once
#include "device_common.h"
#include "layers.h"

namespace rnnt {

namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
// Eight values of a row at their element's alignment (rows of odd length): still one load or store of 16 bytes
typedef bf16x8 bf16x8_any __attribute__((aligned(2)));
typedef f16x8 f16x8_any __attribute__((aligned(2)));
typedef f32x4 f32x4_at4 __attribute__((aligned(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
template <typename T>
struct Vec8;
template <>
struct Vec8<bf16_t> {
    typedef bf16x8 type;
    typedef bf16x8_any any;
};
template <>
struct Vec8<_Float16> {
    typedef f16x8 type;
    typedef f16x8_any any;
};
// Eight floats rounded to 16 bits each, nearest and even (as a vector: two to an instruction)
template <typename T>
__device__ __forceinline__ typename Vec8<T>::type round8(const float (&v)[8]) {
    const f32x8 x = {v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]};
    return __builtin_convertvector(x, typename Vec8<T>::type);
}
// The first `live` of eight consecutive values, zeros for the others
template <typename T>
__device__ __forceinline__ void load8(const T* p, int live, float (&v)[8]) {
    if (live >= 8) {
        if constexpr (sizeof(T) == 2) {
            const typename Vec8<T>::type x = *reinterpret_cast<const typename Vec8<T>::any*>(p);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = (float)x[j];
        } else {
            const f32x4 a = *reinterpret_cast<const f32x4_at4*>(p), b = *reinterpret_cast<const f32x4_at4*>(p + 4);
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
template <typename T>
__device__ __forceinline__ void store8(T* p, int live, const float (&v)[8]) {
    if (live >= 8) {
        if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<typename Vec8<T>::any*>(p) = round8<T>(v);
        } else {
            *reinterpret_cast<f32x4_at4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
            *reinterpret_cast<f32x4_at4*>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < live) p[j] = (T)v[j];
    }
}

// Eight packed 16-bit values, zeros from `live` on
template <typename T>
__device__ __forceinline__ typename Vec8<T>::type take8(const T* p, int live) {
    if (live >= 8) return *reinterpret_cast<const typename Vec8<T>::any*>(p);
    typename Vec8<T>::type x = {};
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < live) x[j] = p[j];
    return x;
}
// The first `live` of eight packed 16-bit values
template <typename T, typename V>
__device__ __forceinline__ void put8(T* p, int live, const V& x) {
    if (live >= 8) *reinterpret_cast<typename Vec8<T>::any*>(p) = x;
    else
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < live) p[j] = x[j];
}

// Eight floats as parts (layers.h) into the four arrays at p.  A finite value that would round to infinity takes the largest bf16 value as its first part.
__device__ __forceinline__ void put_parts8(bf16_t* p, long long part, const float (&v)[8]) {
    bf16x8 h, f, m, l;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float x = v[j];
        const bool finite = fabsf(x) < -RNNT_NEG_INF;
        const float top = __uint_as_float(0x7f7f0000u);
        float hf = (float)(bf16_t)x;
        hf = finite ? __builtin_amdgcn_fmed3f(hf, -top, top) : 0.0f;
        const float r = finite ? x - hf : 0.0f;
        const bf16_t mb = (bf16_t)r;
        h[j] = finite ? (bf16_t)hf : (bf16_t)x;
        f[j] = (bf16_t)hf;
        m[j] = mb;
        l[j] = (bf16_t)(r - (float)mb);
    }
    *reinterpret_cast<bf16x8*>(p) = h;
    *reinterpret_cast<bf16x8*>(p + part) = f;
    *reinterpret_cast<bf16x8*>(p + 2 * part) = m;
    *reinterpret_cast<bf16x8*>(p + 3 * part) = l;
}

// Eight values rounded to bf16 and, where rest is not 0, what that left: bf16 too, at p + rest.  (Nothing is left of an infinity.)
__device__ __forceinline__ void put_rounded8(bf16_t* p, long long rest, const float (&v)[8]) {
    const bf16x8 h = round8<bf16_t>(v);
    *reinterpret_cast<bf16x8*>(p) = h;
    if (rest == 0) return;
    float l[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) l[j] = fabsf((float)h[j]) < -RNNT_NEG_INF ? v[j] - (float)h[j] : 0.0f;
    *reinterpret_cast<bf16x8*>(p + rest) = round8<bf16_t>(l);
}

// Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers, as easy as 1, 2, 3; 2011) with key {seed} on the counter {column / 8, row, offset}:
// the 128 bits of eight columns, 16 for each.
struct RandomBits8 {
    unsigned w[4];
    // entry j's bits in the upper half
    __device__ __forceinline__ unsigned of(int j) const { return (j & 1) ? w[j >> 1] : w[j >> 1] << 16; }
};
__device__ __forceinline__ RandomBits8 random_bits8(unsigned long long seed, unsigned long long offset, unsigned row, unsigned group) {
    unsigned c0 = group, c1 = row, c2 = (unsigned)offset, c3 = (unsigned)(offset >> 32), k0 = (unsigned)seed, k1 = (unsigned)(seed >> 32);
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const unsigned long long p0 = (unsigned long long)c0 * 0xD2511F53u, p1 = (unsigned long long)c2 * 0xCD9E8D57u;
        c0 = (unsigned)(p1 >> 32) ^ c1 ^ k0;
        c1 = (unsigned)p1;
        c2 = (unsigned)(p0 >> 32) ^ c3 ^ k1;
        c3 = (unsigned)p0;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return RandomBits8{{c0, c1, c2, c3}};
}
// Which of columns n .. n + 7 of row m (n a multiple of 8) are kept (d.cut not 0)
__device__ __forceinline__ void keep8(const Dropout& d, long long m, int n, bool (&keep)[8]) {
    const RandomBits8 r = random_bits8(d.state[0], d.state[1], (unsigned)m, (unsigned)n >> 3);
#pragma unroll
    for (int j = 0; j < 8; ++j) keep[j] = r.of(j) >= d.cut << 16;
}
// v[j] *= mask d.scale.  A dropped entry is 0 whatever it was.
__device__ __forceinline__ void drop8(const Dropout& d, const bool (&keep)[8], float (&v)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = keep[j] ? v[j] * d.scale : 0.0f;
}

// FAST: by the exponential and reciprocal instructions (relative error about 1e-6, from |x| = 16 on |x| 6e-8, of tanh see there; results that are rounded to
// bf16); else the math library's functions.
template <bool FAST>
__device__ __forceinline__ float sigmoid(float x) {
    if constexpr (FAST) return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-LOG2E_F * x));
    else return 1.0f / (1.0f + expf(-x));
}
// p, q = sigmoid(+-x), both to their own precision, by one exponential and one reciprocal
template <bool FAST>
__device__ __forceinline__ void sigmoids(float x, float& p, float& q) {
    const float e = FAST ? __builtin_amdgcn_exp2f(-LOG2E_F * fabsf(x)) : expf(-fabsf(x));
    const float most = FAST ? __builtin_amdgcn_rcpf(1.0f + e) : 1.0f / (1.0f + e), least = e * most;
    p = x > 0.0f ? most : least;
    q = x > 0.0f ? least : most;
}
// Phi(-|x|), the normal distribution's tail, and e^{-x^2/2}.  FAST: erfc(z) = t Q(t) e^{-z^2} with t = 1 / (1 + 0.375 z) and a polynomial Q of degree 6
// fitted to it for the smallest relative error over z < 9.3 (6.5e-7; in fp32 2e-6 for |x| < 5, 9e-6 where the tail leaves fp32's range): one reciprocal,
// one exponential.
template <bool FAST>
__device__ __forceinline__ float normal_tail(float x, float& bell) {
    if constexpr (FAST) {
        const float t = __builtin_amdgcn_rcpf(fmaf(0.375f * 0.70710678118654752f, fabsf(x), 1.0f));
        bell = __builtin_amdgcn_exp2f(-0.5f * LOG2E_F * x * x);
        float q = 0.5f * -0.13509601354599f;
        q = fmaf(q, t, 0.5f * 0.3879377841949463f);
        q = fmaf(q, t, 0.5f * -0.12959635257720947f);
        q = fmaf(q, t, 0.5f * 0.2830599546432495f);
        q = fmaf(q, t, 0.5f * 0.1666656881570816f);
        q = fmaf(q, t, 0.5f * 0.2156888246536255f);
        q = fmaf(q, t, 0.5f * 0.21133948862552643f);
        return q * t * bell;
    } else {
        bell = expf(-0.5f * x * x);
        return 0.5f * erfcf(0.70710678118654752f * fabsf(x));
    }
}
// 1 - 2 / (1 + e^{2x}) has an absolute error of 2.4e-7, so near 0 tanh is x itself, which is off by x^2 / 3 of it: 3.1e-5 at most, where the two meet.  Two
// instructions more (16000 x 1024 x 4096: 153.8 us without them, 156.5 with; a series up to x^9 in their place, good to 1e-6, took 10 %).
__device__ __forceinline__ float near_tanh(float x) { return fabsf(x) < 0x1p-7f ? x : fast_tanh(x); }
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
            for (int j = 0; j < 8; ++j) {
                float bell;
                const float q = normal_tail<FAST>(v[j], bell);
                v[j] = v[j] == RNNT_NEG_INF ? 0.0f : v[j] * (v[j] > 0.0f ? 1.0f - q : q);
            }
            break;
        case ACT_TANH:
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = FAST ? near_tanh(v[j]) : tanhf(v[j]);
            break;
        default: break;
    }
}
// A z of +-65504 at most: act' there is its limit, and it times 0 is 0.
__device__ __forceinline__ float bounded(float z) { return __builtin_amdgcn_fmed3f(z, -65504.0f, 65504.0f); }
// g[j] *= act'(z[j]).  NaN where z is (by the functions of z that are not bounded).
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
                float p, q;
                sigmoids<FAST>(z[j], p, q);
                g[j] *= p * fmaf(bounded(z[j]), q, 1.0f);
            }
            break;
        case ACT_GELU:
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float bell;
                const float q = normal_tail<FAST>(z[j], bell);
                g[j] *= fmaf(bounded(z[j]) * 0.3989422804014327f, bell, z[j] > 0.0f ? 1.0f - q : q);
            }
            break;
        case ACT_TANH:
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float p, q;
                sigmoids<FAST>(2.0f * z[j], p, q);                 // 1 - tanh^2 = 4 p q
                g[j] *= 4.0f * p * q;
            }
            break;
        default: break;
    }
}

// A saved pre-activation: fp16 (11 bits, where bf16's eight would add as much to the gradient's error as its own rounding does), beyond its range infinity.
// relu's derivative is its sign: z times 2^127, of which even the smallest nonzero one stays nonzero.  A dropped entry is -infinity: the backward pass need not draw its
// random bits again (16000 x 4096 with gelu': they were half of dz's arithmetic).
__device__ __forceinline__ f16x8 saved8(int act, const float (&z)[8], const Dropout& d, const bool (&keep)[8]) {
    const float up = act == ACT_RELU ? 0x1p127f : 1.0f;
    float s[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) s[j] = z[j] * up;
    if (d.cut != 0)
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j] = keep[j] ? s[j] : RNNT_NEG_INF;
    return round8<_Float16>(s);
}

// ---- what becomes of columns n .. n + 7 (n a multiple of 8) of row m of a product --------------------------------------
__device__ __forceinline__ void load_bias8(const Bias& bias, int n, int N, float (&b)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) b[j] = bias.at(n + j < N ? n + j : N - 1);
}
// (by one workgroup of a launch whose epilogue it is)
__device__ __forceinline__ void pass_rng(const LinearEpilogue& e) {
    if (e.rng_used != nullptr && threadIdx.x < 2) e.rng_used[threadIdx.x] = e.drop.state[threadIdx.x];
}
__device__ __forceinline__ void pass_rng(const StoreEpilogue&) {}
// v: columns n .. n + 7 of row m of the product, with the bias.  fetch: what of memory the epilogue needs (sent ahead of the work on v); factor: what is the
// same for all of a product.
struct LinearStore {
    typedef bf16x8 Extra;
    __device__ static __forceinline__ Extra fetch(const LinearEpilogue& e, long long m, int n) {
        Extra r = bf16x8{0};
        if (e.residual != nullptr && m < e.M && n < e.N) r = take8((const bf16_t*)e.residual + (size_t)m * e.N + n, e.N - n);
        return r;
    }
    __device__ static __forceinline__ float factor(const LinearEpilogue&) { return 1.0f; }
    __device__ static __forceinline__ void store(const LinearEpilogue& e, long long m, int n, float (&v)[8], const Extra& r, float = 1.0f, int = 0) {
        if (m >= e.M || n >= e.N) return;
        const size_t at = (size_t)m * e.N + n;
        bool keep[8] = {};
        if (e.drop.cut != 0) keep8(e.drop, m, n, keep);
        if (e.saved != nullptr) put8((_Float16*)e.saved + at, e.N - n, saved8(e.act, v, e.drop, keep));
        act8<true>(e.act, v);
        if (e.drop.cut != 0) drop8(e.drop, keep, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += (float)r[j];
        put8((bf16_t*)e.y + at, e.N - n, round8<bf16_t>(v));
    }
    __device__ static __forceinline__ void bias(const LinearEpilogue& e, int n, float (&b)[8]) { load_bias8(e.bias, n < e.N ? n : e.N - 1, e.N, b); }
};
struct LinearStore32 {
    typedef f32x8 Extra;
    __device__ static __forceinline__ Extra fetch(const LinearEpilogue& e, long long m, int n) {
        float r[8] = {};
        if (e.residual != nullptr && m < e.M && n < e.N) load8((const float*)e.residual + (size_t)m * e.N + n, e.N - n, r);
        return f32x8{r[0], r[1], r[2], r[3], r[4], r[5], r[6], r[7]};
    }
    __device__ static __forceinline__ float factor(const LinearEpilogue&) { return 1.0f; }
    __device__ static __forceinline__ void store(const LinearEpilogue& e, long long m, int n, float (&v)[8], const Extra& r, float = 1.0f, int = 0) {
        if (m >= e.M || n >= e.N) return;
        const size_t at = (size_t)m * e.N + n;
        bool keep[8] = {};
        if (e.drop.cut != 0) keep8(e.drop, m, n, keep);
        if (e.saved != nullptr) {
            float s[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) s[j] = e.drop.cut == 0 || keep[j] ? v[j] : RNNT_NEG_INF;
            store8((float*)e.saved + at, e.N - n, s);
        }
        act8<false>(e.act, v);
        if (e.drop.cut != 0) drop8(e.drop, keep, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += r[j];
        store8((float*)e.y + at, e.N - n, v);
    }
    __device__ static __forceinline__ void bias(const LinearEpilogue& e, int n, float (&b)[8]) { LinearStore::bias(e, n, b); }
};
struct PlainStore {
    typedef long long Extra;             // the output's row, -1: nowhere
    __device__ static __forceinline__ Extra fetch(const StoreEpilogue& e, long long m, int n) {
        return m >= e.M || n >= e.N ? -1 : e.row_map != nullptr ? (long long)e.row_map[m] : m;
    }
    __device__ static __forceinline__ float factor(const StoreEpilogue& e) { return e.unit != nullptr ? e.scale * *e.unit : e.scale; }
    __device__ static __forceinline__ void store(const StoreEpilogue& e, long long, int n, float (&v)[8], const Extra& x, float factor, int split = 0) {
        if (x < 0) return;
        const size_t at = (size_t)split * e.split_stride + (size_t)x * e.ld + n;
        const int live = e.N - n;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= factor;
        if (e.prev != nullptr) {
            float p[8];
            load8(e.prev + at, live, p);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += p[j];
        }
        if (e.bf16) store8((bf16_t*)e.out + at, live, v);
        else store8((float*)e.out + at, live, v);
    }
    __device__ static __forceinline__ void bias(const StoreEpilogue&, int, float (&b)[8]) {
#pragma unroll
        for (int j = 0; j < 8; ++j) b[j] = 0.0f;
    }
};
// Columns 32 block .. + 31 of a SumJob, by 256 threads in eight rows; the partial sums are added in a fixed order.
__device__ __forceinline__ void sum_parts(const SumJob& j, int blocks, int R, int block, float (*red)[32]) {
    const int c = threadIdx.x & 31, row = threadIdx.x >> 5, n = block * 32 + c;
    if (j.count != nullptr) {
        long long r = (long long)*j.count - j.row0;
        r = r < 0 ? 0 : (r + R - 1) / R;
        blocks = r < blocks ? (int)r : blocks;
    }
    float s = 0.0f;
    if (n < j.N) {
        const float* p = j.part + n;
        int b = row;
        for (; b + 56 < blocks; b += 64) {                         // (eight loads at once: one by one their latency is all there is)
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = p[(size_t)(b + 8 * k) * j.ld];
#pragma unroll
            for (int k = 0; k < 8; ++k) s += v[k];
        }
        for (; b < blocks; b += 8) s += p[(size_t)b * j.ld];
    }
    red[row][c] = s;
    __syncthreads();
    if (row == 0 && n < j.N) {
        float t = 0.0f;
#pragma unroll
        for (int r = 0; r < 8; ++r) t += red[r][c];
        t *= j.unit != nullptr ? j.scale * *j.unit : j.scale;
        if (j.prev != nullptr) t += j.prev[n];
        if (j.bf16) ((bf16_t*)j.out)[n] = (bf16_t)t;
        else ((float*)j.out)[n] = t;
    }
}

template <class E>
struct EpilogueOf;
template <>
struct EpilogueOf<LinearEpilogue> {
    typedef LinearStore type;
};
template <>
struct EpilogueOf<LinearEpilogue32> {
    typedef LinearStore32 type;
};
template <>
struct EpilogueOf<StoreEpilogue> {
    typedef PlainStore type;
};

}  // namespace

}  // namespace rnnt
