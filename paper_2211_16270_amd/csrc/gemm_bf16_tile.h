// bf16 matrix products of the layers beside the transducer loss (device code): C[m, n] = sum_k A(m, k) B(k, n), one output tile per workgroup, what
// becomes of a result is up to an epilogue that is handed eight consecutive columns of a row.
#pragma once
#include "device_common.h"
#include "layers.h"

namespace rnnt {

namespace {

// An operand lies in memory either with k contiguous (KC: element (i, k) at p[i * ld + k]) or with k slow (KS: at p[k * ld + i]); its rows are 16-byte
// aligned.  A stage is 64 of k:
//   KC: [row][64 k], 128 bytes per row, so a copy instruction takes eight whole cache lines; 16-byte granule g of row r lies at place g ^ (r % 8), which
//       spreads the 32 rows of an MFMA fragment's 16-byte reads over all banks;
//   KS: [k][R columns], granule c of row k at place c ^ 4 (k % 4) (conflict-free for the transposing LDS reads that turn it into fragments).
// The copies go global -> LDS without registers.  Rows (KC) or columns (KS) beyond n_i read the last ones again: their results are not
// stored.  Beyond the last k there are zeros: K is a multiple of 64 for KC; the last stage of a KS operand whose K is none is taken from `tail`, 64 rows
// that end in zeros.
constexpr int GK = 64;
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef short s16x8_t __attribute__((ext_vector_type(8)));

// How a product goes over its operands: once; twice, an operand being two bf16 values (GemmOperand::wrap); fp32 values as parts, in pairs.
enum Passes { ONCE = 0, TWICE, IN_PARTS };
// SIDE: 0 A, 1 B
template <int R, bool KS, int WAVES, Passes HOW, int SIDE>
struct TileLoader {
    static constexpr int BYTES = R * GK * 2;
    static constexpr int PW = BYTES / 1024 / WAVES;               // copies per wave and stage
    static constexpr int KR = KS ? 512 / R : 0;                   // rows of k per copy
    static constexpr int NV = KS ? (KR == 2 ? 2 : 1) : PW;
    static_assert(!KS || KR == 2 || KR == 4, "256 or 128 columns");
    static_assert(PW % 2 == 0, "the places of two rows of k repeat every second copy");
    const unsigned char* main;                                    // of this wave's first copy of stage 0
    const unsigned char* tail;
    long long step, ld, part;                                     // bytes
    int last;                                                     // the stage that is read from `tail`, or -1
    int wrap;                                                     // the stage that is stage 0 again
    unsigned voff[NV];

    __device__ __forceinline__ void init(const GemmOperand& o, long long i0, long long n_i, int wave, int lane) {
        ld = o.ld * 2;
        part = o.part * 2;
        last = o.tail != nullptr ? o.tail_stage : -1;
        wrap = o.wrap;
        if constexpr (KS) {
            const int per = R / 8, slot = lane & (per - 1);
            main = (const unsigned char*)o.p + i0 * 2 + (long long)(wave * PW * KR) * ld;
            tail = (const unsigned char*)o.tail + i0 * 2 + (long long)(wave * PW * KR) * ld;
            step = GK * ld;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int dk = lane / per, k = v * KR + dk;
                long long col = i0 + (slot ^ (4 * (k & 3))) * 8;
                col = col < n_i - 8 ? col : n_i - 8;
                voff[v] = (unsigned)(dk * ld + (col - i0) * 2);
            }
        } else {
            main = (const unsigned char*)o.p + i0 * ld;
            tail = nullptr;
            step = GK * 2;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                long long r = i0 + (wave * PW + v) * 8 + (lane >> 3);
                r = r < n_i ? r : n_i - 1;
                voff[v] = (unsigned)((r - i0) * ld + ((lane & 7) ^ (lane >> 3)) * 16);
            }
        }
    }
    // copy t of stage `st` into the operand's LDS area at lds (of this wave's first copy)
    template <int T>
    __device__ __forceinline__ void copy(const unsigned char* st, unsigned lds) const {
        if constexpr (KS) lds_dma16_s(st + (long long)(T * KR) * ld, voff[T % NV], lds + T * 1024);
        else lds_dma16_s(st, voff[T], lds + T * 1024);
    }
    __device__ __forceinline__ const unsigned char* stage(int s) const {
        const unsigned char* p;
        if constexpr (HOW == IN_PARTS) {
            // pairs (1, 3), (2, 2), (3, 1), (1, 2), (2, 1), (0, 0): parts as a table of four bits each
            const int block = s / PAIRS, pair = s - block * PAIRS;
            p = main + block * step + ((SIDE == 0 ? 0x021321u : 0x012123u) >> (4 * pair) & 15u) * part;
        } else if constexpr (HOW == TWICE) {
            const bool again = s >= wrap;
            const int t = again ? s - wrap : s;
            p = (KS && t == last ? tail : main + t * step) + (again ? part : 0);
        } else p = KS && s == last ? tail : main + s * step;
        // (uniform, and said so: the copies take it in scalar registers)
        const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)(size_t)p), hi = __builtin_amdgcn_readfirstlane((unsigned)((size_t)p >> 32));
        size_t u = ((size_t)hi << 32) | lo;
        // (five wait states between a vector instruction that writes a scalar register and the memory instruction that reads it, which the compiler does
        // not add inside assembler text)
        asm volatile("s_nop 4" : "+s"(u));
        return (const unsigned char*)u;
    }
};

// Fragments of one operand, B blocks of 32 rows from i_base (a multiple of 32) on: lane l holds row l % 32, k = 8 (l / 32) .. + 7 of a k16-step.
template <int R, bool KS, int B>
struct TileReader {
    unsigned a[KS ? B : 4];
    __device__ __forceinline__ void init(int i_base, int lane) {
        if constexpr (KS) {
            // transposing read: within 16 lanes, lane 4 j + c supplies 4 columns of row j and lane i receives rows 0..3 of column i
            const int fg = lane >> 4, fj = (lane >> 2) & 3, fc = lane & 3;
#pragma unroll
            for (int b = 0; b < B; ++b) {
                const int col = i_base + 32 * b + 16 * (fg & 1) + 4 * fc;
                a[b] = (unsigned)((8 * (fg >> 1) + fj) * R * 2 + (((col >> 3) ^ (fj << 2)) << 4) + (col & 7) * 2);
            }
        } else {
            const int l32 = lane & 31, hb = lane >> 5;
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) a[kk] = (unsigned)((i_base + l32) * 128 + (((2 * kk + hb) ^ (l32 & 7)) << 4));
        }
    }
    template <int KK, int BLK>
    __device__ __forceinline__ bf16x8 read(const unsigned char* tile) const {
        if constexpr (KS) {
            const unsigned char* p = tile + a[BLK] + KK * 16 * R * 2;
            const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(p));
            const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(p + 4 * R * 2));
            const s16x8_t v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            return __builtin_bit_cast(bf16x8, v);
        } else {
            return *reinterpret_cast<const bf16x8*>(tile + a[KK] + BLK * 32 * 128);
        }
    }
};

// Tile shapes: 256 x 256 with 8 waves (2 x 4, each 128 x 64), one workgroup per compute unit; 128 x 128 with 4 waves (2 x 2, each 64 x 64), two of them.
template <int BM_>
struct TileShape {
    static constexpr int BM = BM_, BN = BM_, WM = 2, WN = BM_ / 64, WAVES = WM * WN, THREADS = 64 * WAVES;
    static constexpr int MT = BM / WM / 32, NT = 2;
    static constexpr unsigned OPER = BM * GK * 2;                 // bytes of one operand's stage
    static constexpr unsigned SMEM = 5 * OPER;                    // three of A's, two of B's
    static constexpr unsigned B_AT = 3 * OPER;
};

// Zeros, or the bias of columns n .. n + 63 (n the same for all lanes) with `beyond` from N on, as they stand in a lane's registers.  Scalar loads: a vector
// load's wait would wait for all the copies sent before it (CE, 1632 rows: 12.9 us, 14.9 with such loads).
struct NoBias {
    __device__ __forceinline__ void operator()(int, int, float (&b)[2][16]) const {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int q = 0; q < 16; ++q) b[j][q] = 0.0f;
    }
};
struct ColumnBias {
    Bias bias;
    int N;
    float beyond;
    __device__ __forceinline__ void operator()(int n, int hb, float (&b)[2][16]) const {
        if (n + 64 > N) {
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int q = 0; q < 16; ++q) {
                    const int c = n + 32 * j + 8 * (q >> 2) + 4 * hb + (q & 3);
                    const float v = bias.at(c < N ? c : N - 1);
                    b[j][q] = c < N ? v : beyond;
                }
        } else if (bias.p == nullptr) {
            NoBias{}(n, hb, b);
        } else if (!bias.bf16) {
            const float __attribute__((address_space(4)))* p = (const float __attribute__((address_space(4)))*)((const float*)bias.p + n);
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int q = 0; q < 16; ++q) {
                    const int c = 32 * j + 8 * (q >> 2) + (q & 3);
                    const float lo = p[c], hi = p[c + 4];
                    b[j][q] = hb ? hi : lo;
                }
        } else {
            const unsigned __attribute__((address_space(4)))* p =
                (const unsigned __attribute__((address_space(4)))*)((const unsigned short*)bias.p + n);
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int q = 0; q < 16; q += 2) {
                    const int c = (32 * j + 8 * (q >> 2) + (q & 3)) / 2;
                    const unsigned lo = p[c], hi = p[c + 2], w = hb ? hi : lo;
                    b[j][q] = __uint_as_float(w << 16);
                    b[j][q + 1] = __uint_as_float(w & 0xffff0000u);
                }
        }
    }
};

// acc[i][j] = the tile's product over the stages [s0, s1): block of 32 rows i of the wave's part, block of 32 columns j.  The matrix instruction takes B's
// fragment first, so lane l holds row l % 32 and register 4 q + r column 8 q + 4 (l / 32) + r.
// LDS holds three stages of A and two of B.  A stage is four k16-steps; the fragments of the next step are read behind the MFMAs of the present one.
// Before the fourth every wave has read all it needs of the stage and the next one has landed: one barrier per stage.  The copies of A two stages ahead
// go out in the first two steps (their buffer became free a stage ago), those of B in the fourth, into the buffer that has just become free.  (Two stages of
// both, all copies in the fourth step: 8192^3 1250 to 1280 TFLOP/s, now 1346 to 1374; without any copies 1470 to 1510.  The rest of the loss is the prologue and
// the epilogue, which nothing hides: 16000 x 1024 x 4096 930 TFLOP/s.)  A wave has priority while it sends MFMAs (11 % of that less without).
// init: what the sums of the columns start from.
// IN_PARTS: the matrix instruction's accumulation rounds towards minus infinity, alike for all results: 5e-11 of a result's size per unit of
// depth, which sums over many of them would show.  So every 1024 of depth the sum changes its sign, and B enters with the other one.
template <class TS, bool AKS, bool BKS, Passes HOW, class INIT>
__device__ __forceinline__ void gemm_tile(f32x16 (&acc)[TS::MT][TS::NT], const GemmOperand& ga, const GemmOperand& gb, long long m0, long long n0,
                                          long long M, long long N, int s0, int s1, unsigned char* smem, const INIT& init) {
    constexpr int MT = TS::MT, NT = TS::NT;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int wm = wave / TS::WN, wn = wave % TS::WN;
    typedef TileLoader<TS::BM, AKS, TS::WAVES, HOW, 0> LA;
    typedef TileLoader<TS::BN, BKS, TS::WAVES, HOW, 1> LB;
    LA la;
    LB lb;
    la.init(ga, m0, M, wave, lane);
    lb.init(gb, n0, N, wave, lane);
    TileReader<TS::BM, AKS, MT> ra;
    TileReader<TS::BN, BKS, NT> rb;
    ra.init(wm * MT * 32, lane);
    rb.init(wn * NT * 32, lane);
    const unsigned base = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)smem;
    const unsigned dst_a = base + (unsigned)(wave * LA::PW) * 1024u, dst_b = base + TS::B_AT + (unsigned)(wave * LB::PW) * 1024u;

    auto start = [&] {
        float b[NT][16];
        init((int)n0 + wn * NT * 32, lane >> 5, b);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int q = 0; q < 16; ++q) acc[i][j][q] = b[j][q];
    };
    if (s0 >= s1) return start();
    const int last = s1 - 1;
    auto issue_a = [&](int s, unsigned buf) {
        const unsigned char* p = la.stage(s);
        static_for<0, LA::PW>([&](auto t) { la.template copy<decltype(t)::value>(p, dst_a + buf); });
    };
    auto issue_b = [&](int s, unsigned buf) {
        const unsigned char* p = lb.stage(s);
        static_for<0, LB::PW>([&](auto t) { lb.template copy<decltype(t)::value>(p, dst_b + buf); });
    };
    bf16x8 fa[2][MT], fb[2][NT];
    issue_a(s0, 0u);
    issue_b(s0, 0u);
    issue_a(s0 < last ? s0 + 1 : last, TS::OPER);
    issue_b(s0 < last ? s0 + 1 : last, TS::OPER);
    start();
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LA::PW + LB::PW) : "memory");
    __syncthreads();
    static_for<0, MT>([&](auto i) { fa[0][decltype(i)::value] = ra.template read<0, decltype(i)::value>(smem); });
    static_for<0, NT>([&](auto j) { fb[0][decltype(j)::value] = rb.template read<0, decltype(j)::value>(smem + TS::B_AT); });

    // the MFMAs of k16-step KK (register set KK % 2); behind them the fragments of the next one are read (at pa, pb) and copies are sent
    auto multiply = [&](auto kk_tag, const unsigned char* pa, const unsigned char* pb, int dma_stage, unsigned dma_buf) {
        constexpr int KK = decltype(kk_tag)::value, set = KK & 1, next = (KK + 1) & 3;
        const unsigned char* src = nullptr;
        if constexpr (KK == 0 || KK == 1) src = la.stage(dma_stage);
        if constexpr (KK == 3) src = lb.stage(dma_stage);
        static_for<0, MT * NT>([&](auto idx_tag) {
            constexpr int idx = decltype(idx_tag)::value, i = idx / NT, j = idx % NT, G = MT * NT;
            if constexpr (idx == 0) __builtin_amdgcn_s_setprio(1);
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[set][j], fa[set][i], acc[i][j], 0, 0, 0);
            // fragments idx * F / G .. of the F = MT + NT of the next step
            constexpr int F = MT + NT, f0 = G >= F ? idx : idx * F / G, f1 = G >= F ? idx + 1 : (idx + 1) * F / G;
            static_for<f0, (f1 < F ? f1 : F)>([&](auto f_tag) {
                constexpr int f = decltype(f_tag)::value;
                if constexpr (f < NT) fb[set ^ 1][f] = rb.template read<next, f>(pb);
                else fa[set ^ 1][f - NT] = ra.template read<next, f - NT>(pa);
            });
            if constexpr (KK == 0 || KK == 1) {
                constexpr int D = LA::PW / 2, d0 = idx * D / G, d1 = (idx + 1) * D / G;
                static_for<d0, d1>([&](auto d) { la.template copy<KK * D + decltype(d)::value>(src, dst_a + dma_buf); });
            }
            if constexpr (KK == 3) {
                constexpr int D = LB::PW, d0 = idx * D / G, d1 = (idx + 1) * D / G;
                static_for<d0, d1>([&](auto d) { lb.template copy<decltype(d)::value>(src, dst_b + dma_buf); });
            }
            if constexpr (idx == G - 1) __builtin_amdgcn_s_setprio(0);
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    unsigned sign = 0;                                            // of B's entries, twice per register
    auto turn_signs = [&](int s) {
        if constexpr (HOW == IN_PARTS) {
            const unsigned now = (s / PAIRS) & (1024 / GK) ? 0x80008000u : 0u;
            if (now != sign) {
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int j = 0; j < NT; ++j) acc[i][j] = -acc[i][j];
                sign = now;
            }
        }
    };
    auto signed_b = [&](int set) {
        if constexpr (HOW == IN_PARTS) {
#pragma unroll
            for (int j = 0; j < NT; ++j) fb[set][j] = __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, fb[set][j]) ^ sign);
        }
    };
    unsigned a0 = 0, a1 = TS::OPER, a2 = 2 * TS::OPER, b0 = 0;    // A's buffers of this stage, the next, the one after; B's of this stage
    for (int s = s0; s < s1; ++s) {
        // (past the end: the last stage again, into buffers nobody reads any more)
        const int ahead = s + 2 < s1 ? s + 2 : last;
        const unsigned char *pa = smem + a0, *pb = smem + TS::B_AT + b0;
        turn_signs(s);
        __builtin_amdgcn_s_waitcnt(WAIT_LGKM0);
        signed_b(0);
        __builtin_amdgcn_sched_barrier(0);
        multiply(std::integral_constant<int, 0>{}, pa, pb, ahead, a2);
        __builtin_amdgcn_s_waitcnt(WAIT_LGKM0);
        signed_b(1);
        __builtin_amdgcn_sched_barrier(0);
        multiply(std::integral_constant<int, 1>{}, pa, pb, ahead, a2);
        __builtin_amdgcn_s_waitcnt(WAIT_LGKM0);
        signed_b(0);
        __builtin_amdgcn_sched_barrier(0);
        multiply(std::integral_constant<int, 2>{}, pa, pb, 0, 0u);
        __builtin_amdgcn_s_waitcnt(WAIT_LGKM0);
        signed_b(1);
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LA::PW) : "memory");       // the next stage has landed; A's after that may be in flight
        __syncthreads();
        __builtin_amdgcn_sched_barrier(0);
        multiply(std::integral_constant<int, 3>{}, smem + a1, smem + TS::B_AT + (b0 ^ TS::OPER), ahead, b0);
        const unsigned t = a0;
        a0 = a1;
        a1 = a2;
        a2 = t;
        b0 ^= TS::OPER;
    }
    if constexpr (HOW == IN_PARTS)
        if (sign != 0) {
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[i][j] = -acc[i][j];
        }
    __builtin_amdgcn_s_waitcnt(WAIT_LGKM0);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");              // no copy may land after this: the epilogue uses LDS
    __syncthreads();
}

// Eight columns of the lane's row: granule p of block j of accumulator d, columns 16 p + 8 (l / 32) .. + 7 of the block
__device__ __forceinline__ void granule8(const f32x16& d, int p, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        unsigned x = __float_as_uint(d[8 * p + i]), y = __float_as_uint(d[8 * p + 4 + i]);
        swap_halves(x, y);
        v[i] = __uint_as_float(x);
        v[4 + i] = __uint_as_float(y);
    }
}
// 32 rows x 64 columns of 16-bit results through 4 KiB of LDS of the wave's own, so that a store covers whole lines: lane l brings granule (j, p) of row
// l % 32 and takes, for t = 0 .. 3, the eight columns 8 (l % 8) .. + 7 of row 8 t + l / 8.  (Granule c of row r at place c xor (r % 8): all banks.)
constexpr unsigned TURN_BYTES = 4096;
__device__ __forceinline__ void turn_put(unsigned char* area, int j, int p, int lane, const u32x4& x) {
    const int row = lane & 31, c = 4 * j + 2 * p + (lane >> 5);
    *reinterpret_cast<u32x4*>(area + row * 128 + ((c ^ (row & 7)) << 4)) = x;
}
__device__ __forceinline__ u32x4 turn_take(const unsigned char* area, int t, int lane) {
    const int row = 8 * t + (lane >> 3);
    return *reinterpret_cast<const u32x4*>(area + row * 128 + (((lane & 7) ^ (row & 7)) << 4));
}
// The same with 32 x 64 fp32 results and 8 KiB: what is done with them is done once per row piece, in a loop.  (16-byte piece c of row r at place
// c xor (r % 16).)
constexpr unsigned TURN32_BYTES = 8192;
__device__ __forceinline__ void turn32_put(unsigned char* area, int j, const f32x16& d, int lane) {
    const int row = lane & 31;
#pragma unroll
    for (int q = 0; q < 4; ++q)
        *reinterpret_cast<f32x4*>(area + row * 256 + (((8 * j + 2 * q + (lane >> 5)) ^ (row & 15)) << 4)) =
            f32x4{d[4 * q], d[4 * q + 1], d[4 * q + 2], d[4 * q + 3]};
}
__device__ __forceinline__ void turn32_take(const unsigned char* area, int t, int lane, float (&v)[8]) {
    const int row = 8 * t + (lane >> 3), c = 2 * (lane & 7);
    const f32x4 a = *reinterpret_cast<const f32x4*>(area + row * 256 + ((c ^ (row & 15)) << 4));
    const f32x4 b = *reinterpret_cast<const f32x4*>(area + row * 256 + (((c + 1) ^ (row & 15)) << 4));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        v[j] = a[j];
        v[4 + j] = b[j];
    }
}
// between the two, and before the area is written again
__device__ __forceinline__ void turn_fence() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Workgroup L -> (split, tile row, tile column).  Workgroups are dealt round-robin to the 8 XCDs, each with its own L2: an XCD takes a contiguous range of
// the tiles, in an order that walks blocks of eight tile columns row by row, so that its 32 compute units share rows of A and columns of B.
struct TilePlace {
    int split, m, n;
};
__device__ __forceinline__ bool place_tile(int L, int mt, int nt, int splits, TilePlace& t) {
    const int tiles = mt * nt, total = tiles * splits, per = (total + 7) >> 3;
    const int w = (L & 7) * per + (L >> 3);
    if ((L >> 3) >= per || w >= total) return false;
    constexpr int GN = 8;
    t.split = w / tiles;
    const int r = w - t.split * tiles, blk = r / (mt * GN), in = r - blk * mt * GN;
    const int nb = nt - blk * GN < GN ? nt - blk * GN : GN;
    t.m = in / nb;
    t.n = blk * GN + in % nb;
    return true;
}

}  // namespace

}  // namespace rnnt
