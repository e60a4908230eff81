// Matrix products of the feed-forward operators: C[m, n] = sum over k of A[m, k] * B[n, k] on the matrix
// instructions, for float32, the two 16-bit types and microscaled 4-bit storage, with what follows the sum
// (biases, gate, activation, rounding) done on the accumulators.
//
// One kernel template for all types, because a 16-byte piece of an operand row is one lane's share of a
// 16x16 matrix instruction in every one of them: 8 values of 16 bits are 16x16x32, 32 values of 4 bits are
// 16x16x128 (and one scale block), and 4 floats feed four 16x16x4.  A tile of K is 128 bytes of a row, two
// such steps.  The order of K inside a tile is free as long as A and B agree.
//
// Operands are brought into LDS by the load that writes there directly (16 bytes a lane, a wavefront's 1024
// bytes in lane order), so the arrangement against bank conflicts is made on the global side: which piece a
// lane fetches.  Two to four K tiles are in LDS: while one is multiplied, the others are on their way.
//
// Layouts.  "K contiguous" (rows of A and B as a linear layer has them): [row][128 bytes], the 16-byte
// piece c of row r at position c ^ (r & 7).  "K strided" (the operands of a gradient, whose sum runs over
// rows): [k][row], read transposed - by the LDS load that transposes 16-bit values, float by float for
// float32 -, in units of 16 rows whose positions are exchanged among the k that one load reads together.
//
// Three kernels: k_big (256 x 256 tiles) for large products, k_mid (64 or 128 x 128) for those of the middle, with K
// shared out and k_join to add the parts where there are few tiles, k_few for a token or a few; alcs_tile_plan.h
// chooses, by what was measured.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <initializer_list>
#include <type_traits>
#include <utility>

#include "alcs_internal.h"
#include "alcs_tile_plan.h"

namespace alcs {
namespace tile {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v2i __attribute__((ext_vector_type(2)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));

// ------------------------------------------------------------------------------ numbers

__device__ inline float to_float(float v) { return v; }
__device__ inline float to_float(__bf16 v) { return (float)v; }
__device__ inline float to_float(_Float16 v) { return (float)v; }
template <int E> struct TypeOf { typedef float type; };
template <> struct TypeOf<kBF16> { typedef __bf16 type; };
template <> struct TypeOf<kF16> { typedef _Float16 type; };

// The gates of alcs.h (alcs_gate).  EXACT: float32 tensors get the library's exponential and division;
// for results of 16 bits the hardware's exp2 and reciprocal are far below the rounding: relative error about (4 + |g|) 2^-24, since
// the exponent's rounding grows with it.
template <bool EXACT> __device__ inline float sigmoid(float g) {
    if (EXACT) return 1.0f / (1.0f + expf(-g));
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g * -1.44269504f));
}
constexpr float kGeluA = 0.7978845608f, kGeluB = 0.044715f;  // sqrt(2/pi)
// GELU's factor (1 + erf(g / sqrt 2)) / 2 and e = exp(-g^2 / 2), the factor as erfc(-g / sqrt 2) / 2: 1 + erf has no digits left
// where it is all but 0 (4 % off at g = -5, nothing right below -5.5).  For 16 bits erfc(x) exp(x^2) = t P(t),
// t = 1 / (1 + 0.428 x), P of degree 7 fitted to the least largest relative error over 0 <= x <= 9.5 (beyond, e is 0): 1e-7,
// and 4e-7 in float32 arithmetic.  Gate gradients of 8192 x 8192 (bfloat16) 123 us, with the library's erfc 155, with erf
// 137; 4096 x 512 -> 2 x 4096 (bfloat16) 52, 67 and 65 us.
template <bool EXACT> __device__ inline float normal_cdf(float g, float &e) {
    if (EXACT) {
        e = expf(-0.5f * g * g);
        return 0.5f * erfcf(g * -0.70710678f);
    }
    e = __builtin_amdgcn_exp2f(g * g * -0.72134752f);
    const float t = __builtin_amdgcn_rcpf(1.0f + 0.3026417f * fabsf(g));
    float p = 0.036575247f;
    p = p * t - 0.15643485f;
    p = p * t + 0.1977404f;
    p = p * t - 0.04732051f;
    p = p * t + 0.12556694f;
    p = p * t + 0.1014797f;
    p = p * t + 0.12170447f;
    p = p * t + 0.12068855f;
    const float q = e * (t * p);
    return g < 0.0f ? q : 1.0f - q;
}
template <bool EXACT> __device__ inline float gate_value(int gate, float g) {
    switch (gate) {
        case ALCS_GATE_RELU: return g < 0.0f ? 0.0f : g;
        case ALCS_GATE_SILU: return g * sigmoid<EXACT>(g);
        case ALCS_GATE_GELU: { float e; return g * normal_cdf<EXACT>(g, e); }
        // 0.5 (1 + tanh z) = sigmoid(2 z)
        case ALCS_GATE_GELU_TANH: return g * sigmoid<EXACT>(2.0f * kGeluA * (g + kGeluB * g * g * g));
        case ALCS_GATE_SIGMOID: return sigmoid<EXACT>(g);
        default: return g;
    }
}
// eight of them: one look at which gate it is
template <bool EXACT> __device__ inline void gate_values(int gate, const float (&g)[8], float (&v)[8]) {
#define ALCS_EACH(kind)                                                        \
    case kind:                                                                 \
        _Pragma("unroll") for (int e = 0; e < 8; ++e) v[e] = gate_value<EXACT>(kind, g[e]); \
        break;
    switch (gate) {
        ALCS_EACH(ALCS_GATE_NONE)
        ALCS_EACH(ALCS_GATE_RELU)
        ALCS_EACH(ALCS_GATE_SILU)
        ALCS_EACH(ALCS_GATE_GELU)
        ALCS_EACH(ALCS_GATE_GELU_TANH)
        ALCS_EACH(ALCS_GATE_SIGMOID)
    }
#undef ALCS_EACH
}
// value and derivative
template <bool EXACT> __device__ inline void gate_both(int gate, float g, float &v, float &d) {
    switch (gate) {
        case ALCS_GATE_RELU: v = g < 0.0f ? 0.0f : g; d = g > 0.0f ? 1.0f : 0.0f; break;
        case ALCS_GATE_SILU: { const float s = sigmoid<EXACT>(g); v = g * s; d = s * (1.0f + g * (1.0f - s)); break; }
        case ALCS_GATE_GELU: {
            float e;
            const float c = normal_cdf<EXACT>(g, e);
            v = g * c;
            d = c + g * 0.3989422804f * e;
            break;
        }
        case ALCS_GATE_GELU_TANH: {
            const float s = sigmoid<EXACT>(2.0f * kGeluA * (g + kGeluB * g * g * g));
            const float b = fminf(g * g, 1e6f);  // beyond it s (1 - s) is 0, and g * g may be infinite
            v = g * s;
            d = s + g * (s * (1.0f - s)) * 2.0f * kGeluA * (1.0f + 3.0f * kGeluB * b);
            break;
        }
        case ALCS_GATE_SIGMOID: v = sigmoid<EXACT>(g); d = v * sigmoid<EXACT>(-g); break;  // (1 - s has no digits left for large g)
        default: v = g; d = 1.0f;
    }
}
template <bool EXACT> __device__ inline void gate_slopes(int gate, const float (&g)[4], float (&v)[4], float (&d)[4]) {
#define ALCS_EACH(kind)                                                        \
    case kind:                                                                 \
        _Pragma("unroll") for (int e = 0; e < 4; ++e) gate_both<EXACT>(kind, g[e], v[e], d[e]); \
        break;
    switch (gate) {
        ALCS_EACH(ALCS_GATE_NONE)
        ALCS_EACH(ALCS_GATE_RELU)
        ALCS_EACH(ALCS_GATE_SILU)
        ALCS_EACH(ALCS_GATE_GELU)
        ALCS_EACH(ALCS_GATE_GELU_TANH)
        ALCS_EACH(ALCS_GATE_SIGMOID)
    }
#undef ALCS_EACH
}
__device__ inline float activate(int act, float v) {
    if (act == ALCS_ACT_NONE) return v;
    v = fmaxf(v, 0.0f);
    return act == ALCS_ACT_RELU6 ? fminf(v, 6.0f) : v;
}

// ------------------------------------------------------------------------------ arguments

struct Operand {
    const char *p;         // first row (K contiguous) or first k (K strided)
    long long pitch;       // bytes from one to the next
    const uint8_t *scales; // kMX4: a byte per 16 bytes of p, rows of pitch / 16
    int rows;              // K strided: elements of a k that may be read, whole pieces
};
struct Args {
    Operand A[2], B[2];  // of the K segments (segs = 2), of the two results (results = 2), or gate and up (B)
    int M, N;            // rows and columns of the result; for a gated product N columns of each projection
    int KA, KB;          // elements of K that A and B hold (A may be padded with zeros beyond B's)
    int segs, results;
    int tiles_m, tiles_n, splits, ktiles;  // ktiles: K tiles of a segment
    unsigned total, per_xcd, xcds;
    float *partial;      // splits > 1: [split][plane][M][sum_pitch(N)] sums
    const float *bias[2];
    void *out[2];        // the result(s); gated: H
    void *pre[2];        // gated: G and U where the caller keeps them, or null
    long long ldo;       // elements from one row of out (and pre) to the next
    int act;             // alcs_activation, or alcs_gate for a gated product
};

__device__ const v4i g_zeros[4] = {};  // what pieces beyond K read

// Direct load of 16 (or 4) bytes a lane from global memory into LDS at lds + lane * 16 (4).  Written out,
// because the compiler would wait for every such load before any later LDS read; here the loads of the next K tile
// stay in flight during the multiply, and wait_loads() stands before the barrier.  (m0 needs one state
// before it is used.)
__device__ inline void lds_load16(const char *g, unsigned lds) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(g), "s"(lds) : "memory");
}
__device__ inline void lds_load4(const char *g, unsigned lds) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(g), "s"(lds) : "memory");
}
__device__ inline void wait_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// an address that is the same for all lanes, in scalar registers
__device__ inline const char *scalar(const char *p) {
    const uintptr_t v = (uintptr_t)p;
    const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)v), hi = __builtin_amdgcn_readfirstlane((unsigned)(v >> 32));
    return (const char *)((uintptr_t)hi << 32 | lo);
}

typedef __attribute__((address_space(3))) char lds_char;
__device__ inline unsigned lds_offset(const char *p) { return (unsigned)(uintptr_t)(lds_char *)(char *)p; }

// ------------------------------------------------------------------------------ one operand's tile

// K strided, 16 bits: what the position of a unit of 16 rows is exchanged with.  A transposing LDS read serves half a
// wavefront at a time, eight k's 32 bytes, which have to lie in different banks; rows of 64 elements (half a turn of the
// banks) differ in the lowest bit of k already.
template <int R> __device__ inline int column_swap(int k) { return R >= 128 ? (k & 3) | (k >> 1 & 4) : (k >> 1 & 1) | (k >> 2 & 2); }

// Where the pieces of R rows (of A, or of B: both projections' for a gated product) and 128 bytes of K lie, brought in by
// four wavefronts.
template <int E, int R, bool KSTRIDED> struct Places {
    static constexpr int W = 4, kElems = per16(E), kLoads = R * kTileBytes / 1024 / W;
    // scales: dwords; of few rows two wavefronts load the same, so that every one has the same number of loads in flight
    static constexpr int kScaleWaves = R * 8 / 256 < W ? R * 8 / 256 : W, kScaleLoads = E == kMX4 ? R * 8 / 256 / kScaleWaves : 0;
    static_assert(R * kTileBytes % (1024 * W) == 0 && (E != kMX4 || R * 8 % (256 * kScaleWaves) == 0), "whole loads per wavefront");

    // K contiguous: the 16 bytes of K that piece c of a row holds.  4-bit: a lane reads pieces c and c + 4, and should
    // find their scales next to each other.
    static __device__ int block_at(int c) { return E == kMX4 ? (c & 3) * 2 + (c >> 2) : c; }
    // where lane `lane`'s piece of load i lies: row of the tile and first k (K contiguous), or k and first row (K strided)
    static __device__ void place(int i, int wave, int lane, int &row, int &k) {
        const int o = (wave * kLoads + i) * 1024 + lane * 16;
        if (!KSTRIDED) {
            row = o / kTileBytes;
            k = block_at(((o / 16) & 7) ^ (row & 7)) * kElems;
        } else {
            constexpr int RB = R * (E == kF32 ? 4 : 2);
            k = o / RB;
            const int piece = (o % RB) / 16;
            if (E == kF32) row = ((piece >> 2) ^ ((k >> 2) & 3)) * 16 + (piece & 3) * 4;
            else row = ((piece >> 1) ^ column_swap<R>(k)) * 16 + (piece & 1) * 8;
        }
    }
};

// A lane's share of 16 rows (from `first` on) in step s of a tile: 16 bytes.
template <int E, int R, bool KSTRIDED> struct Reader {
    int lane;
    int first;
    __device__ Reader(int first_, int lane_) : lane(lane_), first(first_) {}
    __device__ v4i get(const char *lds, int f, int s) const {
        const int r = lane & 15, q = lane >> 4;
        if (!KSTRIDED) {
            return *(const v4i *)(lds + (first + f * 16 + r) * kTileBytes + (((4 * s + q) ^ (r & 7)) << 4));
        }
        constexpr int RB = R * (E == kF32 ? 4 : 2);
        const int u = first / 16 + f;
        if (E == kF32) {
            const char *p = lds + ((4 * s + q) * 4) * RB + ((u ^ q) << 6) + r * 4;
            v4i v;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = *(const int *)(p + j * RB);
            return v;
        }
        const int k = s * 32 + q * 8 + (r >> 2);
        const char *p = lds + k * RB + ((u ^ column_swap<R>(k)) << 5) + (r & 3) * 8;
        typedef __attribute__((address_space(3))) v4s lds_v4s;
        const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s *)(char *)p);
        const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s *)(char *)(p + 4 * RB));
        v4i v;
        __builtin_memcpy(&v, &lo, 8);
        __builtin_memcpy((char *)&v + 8, &hi, 8);
        return v;
    }
};

// c += product of 16 rows of B and 16 rows of A over one step; c[i] of lane (r, q) is the sum for row r
// of A and row 4 q + i of B, so that a lane's four are neighbours in a row of the result.
template <int E> __device__ inline v4f multiply(v4i b, v4i a, v4f c, int s, int sb, int sa) {
    if (E == kBF16) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, b), __builtin_bit_cast(v8bf, a), c, 0, 0, 0);
    } else if (E == kF16) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, b), __builtin_bit_cast(v8h, a), c, 0, 0, 0);
    } else if (E == kF32) {
        const v4f bf = __builtin_bit_cast(v4f, b), af = __builtin_bit_cast(v4f, a);
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(bf[j], af[j], c, 0, 0, 0);
        return c;
    } else {
        const v8i b8 = {b.x, b.y, b.z, b.w, 0, 0, 0, 0}, a8 = {a.x, a.y, a.z, a.w, 0, 0, 0, 0};
        return s == 0 ? __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b8, a8, c, 4, 4, 0, sb, 0, sa)
                      : __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b8, a8, c, 4, 4, 1, sb, 1, sa);
    }
}

// k_big's accumulators: fragment (i, j)'s four values are accumulation registers 4 (8 i + j) and on, by number.  Left
// to itself the compiler moves 256 of them about inside the loop.  Nothing else in that kernel uses accumulation
// registers (tests/test_host_matrix_hazards.py reads that, and the distances below, off the built kernels).
template <int E, int S, int I> __device__ inline void multiply_at(v4i b, v4i a, int sb, int sa) {
    if constexpr (E == kBF16)
        asm volatile("v_mfma_f32_16x16x32_bf16 a[%2:%3], %0, %1, a[%2:%3]" ::"v"(b), "v"(a), "i"(4 * I), "i"(4 * I + 3));
    else if constexpr (E == kF16)
        asm volatile("v_mfma_f32_16x16x32_f16 a[%2:%3], %0, %1, a[%2:%3]" ::"v"(b), "v"(a), "i"(4 * I), "i"(4 * I + 3));
    else if constexpr (S == 0)
        asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 a[%4:%5], %0, %1, a[%4:%5], %2, %3 op_sel_hi:[0,0,0] cbsz:4 blgp:4" ::"v"(b), "v"(a), "v"(sb), "v"(sa), "i"(4 * I), "i"(4 * I + 3));
    else
        asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 a[%4:%5], %0, %1, a[%4:%5], %2, %3 op_sel:[1,1,0] op_sel_hi:[0,0,0] cbsz:4 blgp:4" ::"v"(b), "v"(a), "v"(sb), "v"(sa), "i"(4 * I), "i"(4 * I + 3));
}
template <int I> __device__ inline void clear_at() {
    asm volatile("v_accvgpr_write_b32 a[%0], 0\n\tv_accvgpr_write_b32 a[%1], 0\n\tv_accvgpr_write_b32 a[%2], 0\n\tv_accvgpr_write_b32 a[%3], 0"
                 ::"i"(4 * I), "i"(4 * I + 1), "i"(4 * I + 2), "i"(4 * I + 3));
}
template <int I> __device__ inline v4f read_at() {
    float x, y, z, w;
    asm volatile("v_accvgpr_read_b32 %0, a[%4]\n\tv_accvgpr_read_b32 %1, a[%5]\n\tv_accvgpr_read_b32 %2, a[%6]\n\tv_accvgpr_read_b32 %3, a[%7]"
                 : "=v"(x), "=v"(y), "=v"(z), "=v"(w) : "i"(4 * I), "i"(4 * I + 1), "i"(4 * I + 2), "i"(4 * I + 3));
    return v4f{x, y, z, w};
}
// The kernel has all 256: the registers that are named to the compiler.
#define ALCS_TEN(n) "a" #n "0", "a" #n "1", "a" #n "2", "a" #n "3", "a" #n "4", "a" #n "5", "a" #n "6", "a" #n "7", "a" #n "8", "a" #n "9"
__device__ inline void claim_accumulators() {
    asm volatile("" ::: "a0", "a1", "a2", "a3", "a4", "a5", "a6", "a7", "a8", "a9", ALCS_TEN(1), ALCS_TEN(2), ALCS_TEN(3), ALCS_TEN(4),
                 ALCS_TEN(5), ALCS_TEN(6), ALCS_TEN(7), ALCS_TEN(8), ALCS_TEN(9), ALCS_TEN(10), ALCS_TEN(11), ALCS_TEN(12), ALCS_TEN(13),
                 ALCS_TEN(14), ALCS_TEN(15), ALCS_TEN(16), ALCS_TEN(17), ALCS_TEN(18), ALCS_TEN(19), ALCS_TEN(20), ALCS_TEN(21),
                 ALCS_TEN(22), ALCS_TEN(23), ALCS_TEN(24), "a250", "a251", "a252", "a253", "a254", "a255");
}
#undef ALCS_TEN
// A register that a vector instruction wrote may be a matrix instruction's operand two states later; a matrix
// instruction's result may be read after 19 states, whichever instruction it was.
__device__ inline void operands_ready() { asm volatile("s_nop 1"); }
__device__ inline void matrix_done() { asm volatile("s_nop 15\n\ts_nop 15"); }

// f(0), ..., f(N - 1), each a constant
template <class F, int... I> __device__ inline void each_of(std::integer_sequence<int, I...>, F &&f) { (f(std::integral_constant<int, I>{}), ...); }
template <int N, class F> __device__ inline void each(F &&f) { each_of(std::make_integer_sequence<int, N>{}, f); }

// ------------------------------------------------------------------------------ what follows the sum

// N neighbours, of which `left` are inside the row, in one store (or two of 16 bytes) where all are: of any alignment, which
// the memory system takes.
template <int N, class T> __device__ inline void store_some(T *p, const float *v, int left) {
    T e[N];
#pragma unroll
    for (int i = 0; i < N; ++i) e[i] = (T)v[i];
    if (left >= N) {
        __builtin_memcpy(p, e, sizeof(e));
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < left) p[i] = e[i];
    }
}
template <int N> __device__ inline void load_some(const float *p, float *v, int left) {
    if (left >= N) {
        __builtin_memcpy(v, p, N * sizeof(float));
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < left) v[i] = p[i];
    }
}
// four neighbours of a row: bias, activation, rounding (once, to the result's type)
template <class T> __device__ inline void finish_plain(const Args &a, int result, long long m, int n, v4f c) {
    const int left = a.N - n;
    if (left <= 0) return;
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = activate(a.act, c[i] + (a.bias[0] && i < left ? a.bias[0][n + i] : 0.0f));
    store_some<4>((T *)a.out[result] + m * a.ldo + n, v, left);
}
template <class T> __device__ inline void finish_gated(const Args &a, long long m, int n, v4f g, v4f u) {
    const int left = a.N - n;
    if (left <= 0) return;
    float h[4], gg[4], uu[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        gg[i] = g[i] + (a.bias[0] && i < left ? a.bias[0][n + i] : 0.0f);
        uu[i] = u[i] + (a.bias[1] && i < left ? a.bias[1][n + i] : 0.0f);
        h[i] = gate_value<sizeof(T) == 4>(a.act, gg[i]) * uu[i];
    }
    const long long at = m * a.ldo + n;
    store_some<4>((T *)a.out[0] + at, h, left);
    if (a.pre[0]) {
        store_some<4>((T *)a.pre[0] + at, gg, left);
        store_some<4>((T *)a.pre[1] + at, uu, left);
    }
}

// A wavefront's sums on their way out.  They lie in LDS, rows of COLS floats (of both projections, one behind the
// other, where GATED), the 16-byte piece c of a row at c ^ (row & 7): from there a row leaves in stores of
// neighbouring lanes, whatever its alignment, and the gate is a short loop.  Straight from the accumulators a lane would
// have four values of each of 64 rows' parts: the epilogue of the 128 x 128 tile of an odd-sized product took longer
// than the rest of it.
__device__ inline char *slab_at(char *slab, int pitch, int row, int piece) { return slab + row * pitch + ((piece ^ (row & 7)) << 4); }

template <class T, bool GATED, int COLS, bool SUMS>  // SUMS: K may be shared out
__device__ inline void finish_rows(const Args &a, char *slab, int rows, int m0, int n0, int result, int split, int lane) {
    constexpr bool kExact = sizeof(T) == 4;
    constexpr int kOut = GATED ? COLS / 2 : COLS, kPitch = COLS * 4;
    if (SUMS && a.partial) {  // four neighbours a lane
        constexpr int kLanes = COLS / 4;
        const int piece = lane % kLanes, plane = GATED && piece >= kLanes / 2;
        const int n = n0 + piece % (kOut / 4) * 4, left = a.N - n;
        const long long plane0 = GATED ? split * 2 + plane : (long long)split * a.results + result;
#pragma clang loop unroll_count(2)
        for (int it = 0; it < rows * kLanes / 64; ++it) {
            const int row = it * (64 / kLanes) + lane / kLanes, m = m0 + row;
            const v4f v = *(const v4f *)slab_at(slab, kPitch, row, piece);
            if (m < a.M && left > 0) *(v4f *)(a.partial + (plane0 * a.M + m) * sum_pitch(a.N) + n) = v;
        }
        return;
    }
    constexpr int kLanes = kOut / 8;  // eight neighbours (of both projections) a lane
    const int n = n0 + lane % kLanes * 8, left = a.N - n;
    const bool inside = m0 + rows <= a.M && n0 + kOut <= a.N;  // all of the wavefront's
    float b0[8] = {}, b1[8] = {};
    if (a.bias[0]) load_some<8>(a.bias[0] + n, b0, left);
    if (GATED && a.bias[1]) load_some<8>(a.bias[1] + n, b1, left);
#pragma clang loop unroll_count(2)
    for (int it = 0; it < rows * kLanes / 64; ++it) {
        const int row = it * (64 / kLanes) + lane / kLanes, m = m0 + row;
        float c[8], u[8], h[8];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int piece = lane % kLanes * 2 + k;
            const v4f v = *(const v4f *)slab_at(slab, kPitch, row, piece);
            const v4f w = GATED ? *(const v4f *)slab_at(slab, kPitch, row, piece + COLS / 8) : v;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                c[4 * k + e] = v[e] + b0[4 * k + e];
                u[4 * k + e] = w[e] + b1[4 * k + e];
            }
        }
        const long long at = m * a.ldo + n;
        if (GATED) {
            gate_values<kExact>(a.act, c, h);
#pragma unroll
            for (int e = 0; e < 8; ++e) h[e] *= u[e];
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) h[e] = activate(a.act, c[e]);
        }
        if (inside) {
            store_some<8>((T *)a.out[GATED ? 0 : result] + at, h, 8);
            if (GATED && a.pre[0]) {
                store_some<8>((T *)a.pre[0] + at, c, 8);
                store_some<8>((T *)a.pre[1] + at, u, 8);
            }
        } else if (m < a.M && left > 0) {
            store_some<8>((T *)a.out[GATED ? 0 : result] + at, h, left);
            if (GATED && a.pre[0]) {
                store_some<8>((T *)a.pre[0] + at, c, left);
                store_some<8>((T *)a.pre[1] + at, u, left);
            }
        }
    }
}

// ------------------------------------------------------------------------------ tiles and workgroups

// Tile number `id` of the result: columns of up to 8 tiles of rows at a time, so that neighbouring numbers share
// operands.
__device__ inline void tile_at(const Args &a, unsigned id, int &m, int &n, int &z) {
    const unsigned per = (unsigned)a.tiles_m * a.tiles_n;
    z = (int)(id / per);
    const unsigned t = id % per, strip = t / (8u * a.tiles_n), in = t % (8u * a.tiles_n);
    const unsigned first = strip * 8, rows = min(8u, (unsigned)a.tiles_m - first);
    m = (int)(first + in % rows);
    n = (int)(in / rows);
}
// Workgroups are dealt round-robin to the XCDs: numbers are exchanged such that an XCD works on neighbouring tiles and
// finds their operands in its L2.
__device__ inline bool tile_of(const Args &a, unsigned block, int &m, int &n, int &z) {
    const unsigned id = (block % a.xcds) * a.per_xcd + block / a.xcds;
    if (id >= a.total) return false;
    tile_at(a, id, m, n, z);
    return true;
}

// One operand on its way: aligned, rows at most kNearPitch apart, so that a piece has a 32-bit offset from a base that is
// the same for all lanes and sending for it costs one load and no address arithmetic.
constexpr long long kNearPitch = 1 << 22;
template <int E, int R, bool KSTRIDED> struct NearStage {
    typedef Places<E, R, KSTRIDED> At;
    static constexpr int kElems = At::kElems, kK = 8 * kElems, kLoads = At::kLoads, kScaleLoads = At::kScaleLoads, kScaleWaves = At::kScaleWaves;
    static constexpr int kBias = 3 * 1024;
    unsigned off[kLoads];
    const char *base;  // kBias in front of the tile's first element
    const char *sbase;
    unsigned soff[kScaleLoads ? kScaleLoads : 1];
    template <class F> __device__ void start_rows(int wave, int lane, F row_of, long long pitch) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            int row, k;
            At::place(i, wave, lane, row, k);
            off[i] = (unsigned)row_of(row) * (unsigned)pitch + k / kElems * 16 + kBias - i % 4 * 1024;
        }
    }
    __device__ void start_columns(int wave, int lane, unsigned pitch, int left) {  // left: columns from the tile's first on
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            int row, k;
            At::place(i, wave, lane, row, k);
            off[i] = k * pitch + (unsigned)min(row, left - kElems) * bytes_of(E) + kBias - i % 4 * 1024;
        }
    }
    template <class F> __device__ void start_scales(int wave, int lane, F row_of, long long pitch) {
#pragma unroll
        for (int i = 0; i < kScaleLoads; ++i) {
            const int d = (wave % kScaleWaves * kScaleLoads + i) * 64 + lane;
            soff[i] = (unsigned)row_of(((d >> 7) * 4 + (d & 3)) * 16 + ((d >> 3) & 15)) * (unsigned)(pitch / 16) + ((d >> 2) & 1) * 4;
        }
    }
    // load i of the K tile; WHOLE: all of it inside K, else `left` elements are.  An instruction's own offset moves both its
    // ends, so every fourth load sets the place in LDS (m0) for four, and off[] is relative to `base` - kBias.
    template <bool WHOLE> __device__ void issue(int i, int left, unsigned lds, int wave, int lane) const {
        const unsigned at = lds + (wave * kLoads + i / 4 * 4) * 1024;
        if (WHOLE) {
            if (i % 4 == 0) asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off[i]), "s"(base), "s"(at) : "memory");
            else if (i % 4 == 1) asm volatile("global_load_lds_dwordx4 %0, %1 offset:1024" ::"v"(off[i]), "s"(base) : "memory");
            else if (i % 4 == 2) asm volatile("global_load_lds_dwordx4 %0, %1 offset:2*1024" ::"v"(off[i]), "s"(base) : "memory");
            else asm volatile("global_load_lds_dwordx4 %0, %1 offset:3*1024" ::"v"(off[i]), "s"(base) : "memory");
        } else {
            int row, k, l = lane;
            unsigned o = off[i];
            asm volatile("" : "+v"(l), "+v"(o));  // the last tile's business: nothing of it is kept in registers by the loop
            At::place(i, wave, l, row, k);
            lds_load16(k < left ? base + o + i % 4 * 1024 : (const char *)g_zeros, at + i % 4 * 1024);
        }
    }
    template <bool WHOLE> __device__ void issue_scales(int left, unsigned slds, int wave, int lane) const {
#pragma unroll
        for (int i = 0; i < kScaleLoads; ++i) {
            const unsigned at = slds + (wave % kScaleWaves * kScaleLoads + i) * 256;
            if (WHOLE) asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" ::"v"(soff[i]), "s"(sbase), "s"(at) : "memory");
            else lds_load4(((lane >> 2) & 1) * 128 < left ? sbase + soff[i] : (const char *)g_zeros, at);
        }
    }
};

// Both operands of a BM x BN tile, brought in by four wavefronts (two by two, as they multiply), K tile after K tile.
template <int E, int BM, int BN, bool AK, bool BK, bool GATED> struct Feed {
    static constexpr int kA = BM * kTileBytes, kB = BN * kTileBytes, kSA = E == kMX4 ? BM * 8 : 0, kSB = E == kMX4 ? BN * 8 : 0;
    static constexpr int kBuf = kA + kB + kSA + kSB, kK = 8 * per16(E);
    static constexpr bool kTwo = !AK && BK;  // K in two segments: dX alone
    typedef NearStage<E, BM, AK> StageA;
    typedef NearStage<E, BN, BK> StageB;
    static constexpr int kParts = StageA::kLoads + StageB::kLoads;                             // pieces of issue()
    static constexpr int kInFlight = kParts + StageA::kScaleLoads + StageB::kScaleLoads;       // loads of a K tile
    const Args &a;
    const int wave, lane;
    StageA sa;
    StageB sb;
    int m0, n0, result;
    long long stepA, stepB;
    int next, in_seg;  // the K tile to send for next, counted over the segments, and in its own
    __device__ Feed(const Args &a_, int wave_, int lane_) : a(a_), wave(wave_), lane(lane_) {}

    __device__ void segment(bool second) {
        // nothing that depends on this copy of the lane is computed ahead and kept in registers through the loop
        int l = lane;
        asm volatile("" : "+v"(l));
        const bool sA = second || result == 1;
        const long long pitchA = sA ? a.A[1].pitch : a.A[0].pitch;
        // a gated product's second operand: a wavefront loads rows of one projection
        const bool sB = GATED ? wave & 1 : second;
        const long long pitchB = sB ? a.B[1].pitch : a.B[0].pitch;
        const char *pa = sA ? a.A[1].p : a.A[0].p, *pb = sB ? a.B[1].p : a.B[0].p;
        if (AK) {
            pa += (long long)m0 * bytes_of(E);
            stepA = pitchA * kK;
            sa.start_columns(wave, l, (unsigned)pitchA, a.A[0].rows - m0);
        } else {
            pa += m0 * pitchA;
            stepA = kTileBytes;
            sa.start_rows(wave, l, [&](int row) { return min(row, a.M - 1 - m0); }, pitchA);
        }
        if (BK) {
            pb += (long long)n0 * bytes_of(E);
            stepB = pitchB * kK;
            sb.start_columns(wave, l, (unsigned)pitchB, a.B[0].rows - n0);
        } else {
            pb += n0 * pitchB;
            stepB = kTileBytes;
            // a wavefront's columns: half of them of the gate, half of the other projection
            sb.start_rows(wave, l, [&](int row) { return min(GATED ? row / (BN / 2) * (BN / 4) + row % (BN / 4) : row, a.N - 1 - n0); }, pitchB);
        }
        sa.base = scalar(pa + in_seg * stepA - StageA::kBias);
        sb.base = scalar(pb + in_seg * stepB - StageB::kBias);
        if (E == kMX4) {
            sa.start_scales(wave, l, [&](int row) { return min(row, a.M - 1 - m0); }, pitchA);
            sb.start_scales(wave, l, [&](int row) { return min(row, a.N - 1 - n0); }, pitchB);
            sa.sbase = scalar((const char *)a.A[0].scales + m0 * (pitchA / 16) + in_seg * 8);
            sb.sbase = scalar((const char *)a.B[0].scales + n0 * (pitchB / 16) + in_seg * 8);
        }
    }
    // tile (tm, tn) of result z, from K tile `from` on
    __device__ void begin(int tm, int tn, int z, int from) {
        m0 = tm * BM;
        n0 = tn * (GATED ? BN / 2 : BN);
        result = z;
        next = from;
        const int s = kTwo && from >= a.ktiles;
        in_seg = from - s * a.ktiles;
        segment(s);
    }
    // one part of the loads of K tile `next`
    template <bool WHOLE> __device__ void issue(int part, unsigned to) const {
        const int leftA = a.KA - in_seg * kK, leftB = a.KB - in_seg * kK;
        if (part < StageA::kLoads) sa.template issue<WHOLE>(part, leftA, to, wave, lane);
        else sb.template issue<WHOLE>(part - StageA::kLoads, leftB, to + kA, wave, lane);
    }
    template <bool WHOLE> __device__ void issue_scales(bool of_b, unsigned to) const {
        if (E != kMX4) return;
        if (of_b) sb.template issue_scales<WHOLE>(a.KB - in_seg * kK, to + kA + kB + kSA, wave, lane);
        else sa.template issue_scales<WHOLE>(a.KA - in_seg * kK, to + kA + kB, wave, lane);
    }
    __device__ void issued(int end) {
        sa.base = scalar(sa.base + stepA);
        sb.base = scalar(sb.base + stepB);
        if (E == kMX4) { sa.sbase = scalar(sa.sbase + 8); sb.sbase = scalar(sb.sbase + 8); }
        ++next;
        ++in_seg;
        if constexpr (kTwo) {
            if (in_seg == a.ktiles && next < end) {
                in_seg = 0;
                segment(true);
            }
        }
    }
    __device__ bool whole() const { return (in_seg + 1) * kK <= min(a.KA, a.KB); }
    __device__ void issue_all(unsigned to, int end) {
        if (whole()) {
#pragma unroll
            for (int part = 0; part < kParts; ++part) issue<true>(part, to);
            issue_scales<true>(false, to);
            issue_scales<true>(true, to);
        } else {
#pragma unroll
            for (int part = 0; part < kParts; ++part) issue<false>(part, to);
            issue_scales<false>(false, to);
            issue_scales<false>(true, to);
        }
        issued(end);
    }
};

// ------------------------------------------------------------------------------ small tiles

// BM x 128 (64 or 128 rows), NS K tiles in LDS.  A K tile is two steps; the fragments of the next step are read and the
// pieces of a later tile sent for between the matrix instructions of this one, so that a wavefront waits for neither.
// One barrier a tile, in front of its second step, as in k_big.  Two workgroups share a compute unit; 128 rows whose
// tiles are no more than the card has units have all of its LDS, and with four K tiles there the weights of a deep product
// arrive as fast as memory has them: 65 x 4096 -> 2 x 16384 (bfloat16) 44 us (6.2 TB/s), with two 62; 256 x 4096 ->
// 2 x 8192 39 and 47.  (Of 16 K tiles, 512 x 1024 -> 2 x 4096, two are faster: 13.2 us, four 13.7.)
template <int E, class T, int BM, int NS, bool AK, bool BK, bool GATED> __device__ __forceinline__ void mid_tile(const Args &a, unsigned block, char *lds) {
    typedef Feed<E, BM, 128, AK, BK, GATED> Feeds;
    constexpr int FM = BM / 32, FN = 4, kA = Feeds::kA, kB = Feeds::kB, kSA = Feeds::kSA, kBuf = Feeds::kBuf;
    constexpr int kSlots = FM * FN, kReads = FM + FN;
    int tm, tn, z;
    if (!tile_of(a, block, tm, tn, z)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave >> 1, wn = wave & 1;
    const int result = a.results == 2 ? z & 1 : 0, split = a.results == 2 ? z >> 1 : z;
    const int all = a.ktiles * a.segs;
    const int from = (int)((long long)all * split / a.splits), to = (int)((long long)all * (split + 1) / a.splits);
    const unsigned lds0 = lds_offset(lds);
    Feeds feed(a, wave, lane);
    feed.begin(tm, tn, result, from);
#pragma unroll
    for (int k = 0; k < NS; ++k)
        if (from + k < to) feed.issue_all(lds0 + k * kBuf, to);
    const Reader<E, BM, AK> ra(wm * FM * 16, lane);
    const Reader<E, 128, BK> rb(wn * FN * 16, lane);
    v4f acc[FM][FN] = {};
    v4i fa[2][FM], fb[2][FN];
    int ca[2][FM] = {}, cb[2][FN] = {};  // scales of this tile, [1]: of the next
    const int scale_at = ((lane & 15) * 2 + (lane >> 5)) * 16, shift = lane & 16;
    auto read_scales = [&](const char *here, int into) {
        if (E != kMX4) return;
        const char *p = here + kA + kB + scale_at;
        const v4i va = *(const v4i *)(p + wm * FM / 4 * 512), vb = *(const v4i *)(p + kSA + wn * 512);
#pragma unroll
        for (int j = 0; j < FM; ++j) ca[into][j] = (unsigned)(FM == 2 && wm & 1 ? va[(2 + j) & 3] : va[j]) >> shift;
#pragma unroll
        for (int j = 0; j < FN; ++j) cb[into][j] = (unsigned)vb[j] >> shift;
    };
    // K tile t's loads, while those of the ones behind it may still be on their way
    auto arrived = [&](int t) {
        if (NS >= 3 && t + NS - 2 < to) asm volatile("s_waitcnt vmcnt(%0)" ::"i"((NS - 2) * Feeds::kInFlight) : "memory");
        else wait_loads();
    };
    if (from + NS - 1 < to) asm volatile("s_waitcnt vmcnt(%0)" ::"i"((NS - 1) * Feeds::kInFlight) : "memory");
    else wait_loads();
    __syncthreads();
#pragma unroll
    for (int f = 0; f < FN; ++f) fb[0][f] = rb.get(lds + kA, f, 0);
#pragma unroll
    for (int f = 0; f < FM; ++f) fa[0][f] = ra.get(lds, f, 0);
    read_scales(lds, 0);
    for (int t = from, buf = 0; t < to; ++t) {
        char *here = lds + buf * kBuf;
        const unsigned free = lds0 + buf * kBuf;
        buf = buf + 1 == NS ? 0 : buf + 1;
        char *there = lds + buf * kBuf;
        bool whole = false;
        auto step = [&](auto which) {
            constexpr int S = decltype(which)::value;
            each<kSlots>([&](auto slot) {
                constexpr int at = decltype(slot)::value, i = at / FN, j = at % FN;
                acc[i][j] = multiply<E>(fb[S][j], fa[S][i], acc[i][j], S, E == kMX4 ? cb[0][j] : 0, E == kMX4 ? ca[0][i] : 0);
                // (behind the last tile the fragments are those of an old one, and nobody multiplies them)
                char *src = S == 0 ? here : there;
                if constexpr (at < FN) fb[1 - S][at] = rb.get(src + kA, at, 1 - S);
                else if constexpr (at < kReads) fa[1 - S][at - FN] = ra.get(src, at - FN, 1 - S);
                if constexpr (S == 1 && at < Feeds::kParts)
                    if (whole) {
                        feed.template issue<true>(at, free);
                        if (at == Feeds::kParts - 1) {
                            feed.template issue_scales<true>(false, free);
                            feed.template issue_scales<true>(true, free);
                        }
                    }
                if constexpr (S == 1 && at == kSlots - 2) read_scales(there, 1);
                __builtin_amdgcn_sched_barrier(0);
            });
        };
        step(std::integral_constant<int, 0>{});
        arrived(t + 1);
        __syncthreads();  // the next tile is there, and nobody reads this one any more
        const bool more = feed.next < to;
        whole = more && feed.whole();
        if (more && !whole) feed.issue_all(free, to);
        step(std::integral_constant<int, 1>{});
        if (whole) feed.issued(to);
#pragma unroll
        for (int j = 0; j < FM; ++j) ca[0][j] = ca[1][j];
#pragma unroll
        for (int j = 0; j < FN; ++j) cb[0][j] = cb[1][j];
    }
    __syncthreads();
    char *slab = lds + wave * (FM * FN * 1024);
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) *(v4f *)slab_at(slab, FN * 64, i * 16 + (lane & 15), j * 4 + (lane >> 4)) = acc[i][j];
    finish_rows<T, GATED, FN * 16, true>(a, slab, FM * 16, feed.m0 + wm * FM * 16, feed.n0 + wn * (GATED ? FN / 2 : FN) * 16, result, split, lane);
}
template <int E, class T, int BM, int NS, bool AK, bool BK, bool GATED> __global__ __launch_bounds__(256, 2) void k_mid(const Args a) {
    extern __shared__ __align__(16) char lds[];
    mid_tile<E, T, BM, NS, AK, BK, GATED>(a, blockIdx.x, lds);
}
constexpr int stages_of(int BM) { return BM == 64 ? 3 : 2; }  // of two workgroups on a compute unit

// The sums that the gradients at the gate were left in, by parts of the rows: 32 columns and eight shares of the parts a
// workgroup, each added in the order of the parts, the shares in theirs.
struct BiasArgs {
    const float *sums;  // [part][2][F]
    int parts, F;
    void *dbg, *dbu;
    unsigned blocks;
};
template <class T> __device__ inline void bias_tile(const BiasArgs &a, unsigned block, float *lds) {
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    const long long at = (long long)block * 32 + x;
    float s = 0.0f;
    if (at < 2LL * a.F) {
        const int from = (int)((long long)a.parts * y / 8), to = (int)((long long)a.parts * (y + 1) / 8);
#pragma clang loop unroll_count(8)
        for (int k = from; k < to; ++k) s += a.sums[(long long)k * 2 * a.F + at];
    }
    lds[y * 32 + x] = s;
    __syncthreads();
    if (y || at >= 2LL * a.F) return;
#pragma unroll
    for (int k = 1; k < 8; ++k) s += lds[k * 32 + x];
    T *out = (T *)(at < a.F ? a.dbg : a.dbu);
    if (out) out[at % a.F] = (T)s;
}

// A layer's gradients in one launch: dX (K strided in B) and dW (in both), which alone do not fill the card where there
// are few tiles, and the biases'.  The product whose workgroups take longer is the first; nx, nw: its workgroups, a
// multiple of the XCDs.
template <int E, class T, int BMX, int BMW>
__global__ __launch_bounds__(256, 2) void k_pair(const Args x, const Args w, const BiasArgs b, unsigned nx, unsigned nw, int x_first) {
    extern __shared__ __align__(16) char lds[];
    const unsigned block = blockIdx.x;
    if (block >= nx + nw) bias_tile<T>(b, block - nx - nw, (float *)lds);
    else if (x_first ? block < nx : block >= nw) mid_tile<E, T, BMX, stages_of(BMX), false, true, false>(x, block - (x_first ? 0 : nw), lds);
    else mid_tile<E, T, BMW, stages_of(BMW), true, true, false>(w, block - (x_first ? nx : 0), lds);
}

// ------------------------------------------------------------------------------ large tiles

// 256 x 256, four wavefronts with 128 x 128 each, one per SIMD: what LDS has to deliver falls with the
// wavefront's tile (at 128 x 64 its reads and the arriving tiles take as many cycles as the matrix instructions).
// With one wavefront a SIMD nothing else fills its waits, so the loop is laid out by hand: a K tile is two
// steps of 64 matrix instructions, and during each the fragments of the next step are read.  One barrier a
// tile, in front of its second step: by then every wavefront has read this tile to its end and the next one has
// arrived, so the one after that can be sent for into this tile's buffer, a whole tile ahead.
constexpr int kBigSide = 256;

// A workgroup takes tile after tile: the next one's first K tile is on its way while this one's result leaves.
template <int E, class T, bool AK, bool BK, bool GATED> __global__ __launch_bounds__(256, 1) void k_big(const Args a) {
    typedef Feed<E, kBigSide, kBigSide, AK, BK, GATED> Feeds;
    constexpr int kA = Feeds::kA, kS = Feeds::kSA, kBuf = Feeds::kBuf;
    extern __shared__ __align__(16) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave >> 1, wn = wave & 1;
    const int all = a.ktiles * a.segs;
    const unsigned first = blockIdx.x % a.xcds * a.per_xcd, end = min(first + a.per_xcd, a.total);
    unsigned id = first + blockIdx.x / a.xcds;
    if (id >= end) return;
    claim_accumulators();
    const unsigned lds0 = lds_offset(lds);
    Feeds feed(a, wave, lane);
    auto begin = [&](unsigned tile) {
        int tm, tn, z;
        tile_at(a, tile, tm, tn, z);
        feed.begin(tm, tn, a.results == 2 ? z : 0, 0);
    };
    const Reader<E, kBigSide, AK> ra(wm * 128, lane);
    const Reader<E, kBigSide, BK> rb(wn * 128, lane);
    v4i pa[8], pb[8], qa[8], qb[8];  // fragments of a first and of a second step
    // A tile's scales, step s takes byte s: as they lie in LDS, shifted for the first step, and a copy of those for the
    // second (while it runs, the next tile's come in).
    v4i raw[4] = {};
    int ca[8] = {}, cb[8] = {}, da[8] = {}, db[8] = {};
    const int scale_at = ((lane & 15) * 2 + (lane >> 5)) * 16, shift = lane & 16;
    auto read_scales = [&](const char *here, int k) {
        const char *p = here + 2 * kA + scale_at + (k & 1) * 512;
        raw[k] = *(const v4i *)(k < 2 ? p + wm * 1024 : p + kS + wn * 1024);
    };
    auto shift_scale = [&](int k) {
        int &c = k < 8 ? ca[k & 7] : cb[k & 7];
        asm volatile("v_lshrrev_b32 %0, %1, %2" : "=v"(c) : "v"(shift), "v"(raw[k / 4][k & 3]));
    };
    auto copy_scale = [&](int k) {
        int &d = k < 8 ? da[k & 7] : db[k & 7];
        asm volatile("v_mov_b32 %0, %1" : "=v"(d) : "v"(k < 8 ? ca[k & 7] : cb[k & 7]));
    };
    // A wavefront issues in order, and a matrix instruction keeps its unit busy for four issues: one other
    // instruction fits behind each without a gap, several in a row do not.  Neighbouring instructions share an
    // operand, also from one row of fragments to the next (the columns go to and fro): fewer registers change.
    bool ready = false;  // a K tile is left to send for, and all of it lies inside K
    auto first_step = [&](const char *here) {
        operands_ready();
        each<64>([&](auto k) {
            constexpr int at = decltype(k)::value, i = at / 8, j = i % 2 ? 7 - at % 8 : at % 8;
            multiply_at<E, 0, i * 8 + j>(pb[j], pa[i], cb[j], ca[i]);
            if constexpr (at < 32 && at % 4 == 0) qb[at / 4] = rb.get(here + kA, at / 4, 1);
            if constexpr (at < 32 && at % 4 == 2) qa[at / 4] = ra.get(here, at / 4, 1);
            if constexpr (E == kMX4 && at >= 40 && at < 56) copy_scale(at - 40);
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    // (behind the last tile the fragments read are those of an old one, and nobody multiplies them)
    auto second_step = [&](auto load, const char *there, unsigned to) {
        operands_ready();
        each<64>([&](auto k) {
            constexpr int at = decltype(k)::value, i = at / 8, j = i % 2 ? 7 - at % 8 : at % 8;
            multiply_at<E, 1, i * 8 + j>(qb[j], qa[i], db[j], da[i]);
            if constexpr (at < 32 && at % 4 == 0) pb[at / 4] = rb.get(there + kA, at / 4, 0);
            if constexpr (at < 32 && at % 4 == 2) pa[at / 4] = ra.get(there, at / 4, 0);
            // (early, but for transposing reads, which are twice as many: spread over the step)
            constexpr int every = AK || BK ? 4 : 2;
            if constexpr (decltype(load)::value) {
                if constexpr (at % every == every - 1 && at / every < 16) feed.template issue<true>(at / every, to);
                if constexpr (at == 37 || at == 41) feed.template issue_scales<true>(at == 41, to);
                if constexpr (at == (every == 4 ? 63 : 54)) feed.issued(all);
                if constexpr (at == (every == 4 ? 63 : 58)) ready = feed.next < all && feed.whole();
            }
            if constexpr (E == kMX4 && at >= 32 && at < 36) read_scales(there, at - 32);
            if constexpr (E == kMX4 && at >= 46 && at < 62) shift_scale(at - 46);
            __builtin_amdgcn_sched_barrier(0);
        });
    };

    begin(id);
    feed.issue_all(lds0, all);
    for (;;) {
        if (feed.next < all) {
            feed.issue_all(lds0 + kBuf, all);
            asm volatile("s_waitcnt vmcnt(%0)" ::"i"(Feeds::kInFlight) : "memory");  // the first K tile's, and everything before
        } else {
            wait_loads();
        }
        __syncthreads();
#pragma unroll
        for (int f = 0; f < 8; ++f) {
            pa[f] = ra.get(lds, f, 0);
            pb[f] = rb.get(lds + kA, f, 0);
        }
        if (E == kMX4) {
#pragma unroll
            for (int k = 0; k < 4; ++k) read_scales(lds, k);
#pragma unroll
            for (int k = 0; k < 16; ++k) shift_scale(k);
        }
        each<64>([&](auto k) { clear_at<decltype(k)::value>(); });
        ready = feed.next < all && feed.whole();
        for (int t = 0; t < all; ++t) {
            char *here = lds + (t & 1) * kBuf, *there = lds + (~t & 1) * kBuf;
            first_step(here);
            wait_loads();
            __syncthreads();
            const unsigned to = lds0 + (t & 1) * kBuf;
            if (ready) {
                second_step(std::true_type{}, there, to);
            } else {
                if (feed.next < all) feed.issue_all(to, all);
                ready = feed.next < all && feed.whole();
                second_step(std::false_type{}, there, to);
            }
        }
        matrix_done();
        __syncthreads();  // nobody reads LDS any more
        const int m = feed.m0 + wm * 128, n = feed.n0 + wn * (GATED ? 64 : 128), which = feed.result;
        id += gridDim.x / a.xcds;
        const bool more = id < end;
        if (more) {
            begin(id);
            feed.issue_all(lds0, all);
        }
        // 16 KB of LDS of the wavefront's own, 32 rows at a time
        int l = lane;
        asm volatile("" : "+v"(l));
        char *slab = lds + kBuf + wave * 16384;
#pragma clang loop unroll(disable)
        for (int quarter = 0; quarter < 4; ++quarter) {
            each<4>([&](auto which_quarter) {  // a register has no number that a loop could count
                if (quarter != which_quarter) return;
                each<16>([&](auto k) {
                    constexpr int i = decltype(k)::value / 8, j = decltype(k)::value % 8;
                    const int row = i * 16 + (l & 15);
                    *(v4f *)slab_at(slab, 512, row, j * 4 + (l >> 4)) = read_at<(decltype(which_quarter)::value * 2 + i) * 8 + j>();
                });
            });
            finish_rows<T, GATED, 128, false>(a, slab, 32, m + quarter * 32, n, which, 0, l);
        }
        if (!more) break;
        __syncthreads();
    }
}

// The sums of a split K, added in the order of the splits; a thread has four neighbours of a row.
template <class T, bool GATED> __global__ __launch_bounds__(256) void k_join(const Args a) {
    const int quads = (a.N + 3) / 4;
    const unsigned at = blockIdx.x * 256 + threadIdx.x;
    const int planes = GATED ? 1 : a.results;
    if (at >= (long long)planes * a.M * quads) return;
    const int n = (int)(at % (unsigned)quads) * 4;
    const long long row = at / (unsigned)quads;  // plane * M + m
    const int pitch = sum_pitch(a.N);
    const long long plane = (long long)(GATED ? 2 : a.results) * a.M * pitch;
    v4f s[2] = {};
#pragma clang loop unroll_count(4)
    for (int k = 0; k < a.splits; ++k)
#pragma unroll
        for (int h = 0; h < (GATED ? 2 : 1); ++h) s[h] += *(const v4f *)(a.partial + k * plane + (row + (long long)h * a.M) * pitch + n);
    if (GATED) finish_gated<T>(a, row, n, s[0], s[1]);
    else finish_plain<T>(a, (int)(row / a.M), row % a.M, n, s[0]);
}

// ------------------------------------------------------------------------------ few rows

// 16 * MF rows of A (a token, a few requests) a workgroup: the weights are read once and the product is bound by
// their bytes, so nothing is staged.  Operands of any alignment and distance, and so also the way of many rows whose
// operands the tiles do not take, where there is no room for copies.  A workgroup has 16 columns (of both projections
// where GATED); its wavefronts share out K in pieces of 256 bytes a row, read their fragments straight from memory,
// four steps ahead of the multiply, and add their sums through LDS in a fixed order.  Rows of A beyond M read the last
// row.
template <int E, bool ALIGNED> __device__ inline v4i piece_of(const char *row, int k, int K) {
    constexpr int kElems = per16(E);
    v4i v = {0, 0, 0, 0};
    if (ALIGNED) {
        if (k < K) v = *(const v4i *)(row + (long long)(k / kElems) * 16);
    } else {
        typedef typename TypeOf<E>::type T;
        const char *p = row + (long long)k * bytes_of(E);
        if (k + kElems <= K) {
            __builtin_memcpy(&v, p, 16);
        } else if (k < K) {
            T e[kElems] = {};
#pragma unroll
            for (int j = 0; j < kElems; ++j)
                if (k + j < K) __builtin_memcpy(&e[j], p + j * sizeof(T), sizeof(T));
            __builtin_memcpy(&v, e, 16);
        }
    }
    return v;
}

template <int E, class T, int MF, bool GATED, bool ALIGNED>
__global__ __launch_bounds__(512, 2) void k_few(const Args a) {
    constexpr int kElems = per16(E), P = GATED ? 2 : 1;
    extern __shared__ __align__(16) char lds[];  // [wavefront][plane][MF][64] v4f
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), W = blockDim.x >> 6;
    const unsigned across = (unsigned)(a.N + 15) / 16;
    const int r = lane & 15, q = lane >> 4, n0 = (int)(blockIdx.x % across) * 16, m0 = (int)(blockIdx.x / across) * 16 * MF;
    const int n = min(n0 + r, a.N - 1);
    const char *w[P];
#pragma unroll
    for (int p = 0; p < P; ++p) w[p] = a.B[p].p + n * a.B[p].pitch;
    const char *x[MF];
    const char *xs[MF], *ws = nullptr;
#pragma unroll
    for (int f = 0; f < MF; ++f) {
        const int m = min(m0 + f * 16 + r, a.M - 1);
        x[f] = a.A[0].p + m * a.A[0].pitch;
        if (E == kMX4) xs[f] = (const char *)a.A[0].scales + m * (a.A[0].pitch / 16);
    }
    if (E == kMX4) ws = (const char *)a.B[0].scales + n * (a.B[0].pitch / 16);
    v4f acc[P][MF] = {};
    const int K = a.KA;
    for (int k0 = wave * 16 * kElems; k0 < K; k0 += W * 16 * kElems) {
        v4i fw[P][4], fx[MF][4];
        int sw = 0, sx[MF];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            // 4-bit: a lane takes four neighbouring blocks, whose scales are one dword
            const int k = k0 + (E == kMX4 ? 4 * q + s : 4 * s + q) * kElems;
#pragma unroll
            for (int p = 0; p < P; ++p) fw[p][s] = piece_of<E, ALIGNED>(w[p], k, K);
#pragma unroll
            for (int f = 0; f < MF; ++f) fx[f][s] = piece_of<E, ALIGNED>(x[f], k, K);
        }
        if (E == kMX4) {
            const int at = k0 / 32 + 4 * q, in = k0 + 4 * q * 32 < K;
            sw = in ? *(const int *)(ws + at) : 0;
#pragma unroll
            for (int f = 0; f < MF; ++f) sx[f] = in ? *(const int *)(xs[f] + at) : 0;
        }
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int f = 0; f < MF; ++f) {
                    if (E == kMX4) {
                        acc[p][f] = multiply<E>(fw[p][s], fx[f][s], acc[p][f], 0, (unsigned)sw >> (8 * s), (unsigned)sx[f] >> (8 * s));
                    } else {
                        acc[p][f] = multiply<E>(fw[p][s], fx[f][s], acc[p][f], 0, 0, 0);
                    }
                }
    }
    v4f *mine = (v4f *)lds + (size_t)wave * P * MF * 64;
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int f = 0; f < MF; ++f) mine[(p * MF + f) * 64 + lane] = acc[p][f];
    __syncthreads();
    for (int f = wave; f < MF; f += W) {
        v4f s[P] = {};
        for (int k = 0; k < W; ++k)
#pragma unroll
            for (int p = 0; p < P; ++p) s[p] += ((const v4f *)lds)[((size_t)k * P * MF + p * MF + f) * 64 + lane];
        const int m = m0 + f * 16 + r;
        if (m < a.M) {
            if (GATED) finish_gated<T>(a, m, n0 + q * 4, s[0], s[P - 1]);
            else finish_plain<T>(a, 0, m, n0 + q * 4, s[0]);
        }
    }
}

// ------------------------------------------------------------------------------ launches

inline int launched() {
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return ALCS_OK;
    set_hip_error((int)e);
    return ALCS_E_HIP;
}

template <int E, class T, int BM, int NS, bool AK, bool BK, bool GATED> int launch_mid(Args &a, hipStream_t stream) {
    constexpr int lds = NS * Feed<E, BM, 128, AK, BK, GATED>::kBuf;
    static_assert(lds <= (NS > 3 ? 160 : 80) * 1024, "two workgroups on a compute unit, one where NS is more than 3");
    auto kern = k_mid<E, T, BM, NS, AK, BK, GATED>;
    const int rc = allow_lds((const void *)kern, lds);
    if (rc != ALCS_OK) return rc;
    hipLaunchKernelGGL(kern, dim3(a.per_xcd * a.xcds), dim3(256), lds, stream, a);
    return launched();
}
template <int E, class T, bool AK, bool BK, bool GATED> int launch_big(Args &a, int cus, hipStream_t stream) {
    constexpr int lds = 4 * (kBigSide * kTileBytes + (E == kMX4 ? kBigSide * 8 : 0));
    auto kern = k_big<E, T, AK, BK, GATED>;
    const int rc = allow_lds((const void *)kern, lds);
    if (rc != ALCS_OK) return rc;
    const unsigned share = std::max(1, cus / (int)a.xcds);  // one workgroup per compute unit
    hipLaunchKernelGGL(kern, dim3(std::min(a.per_xcd, share) * a.xcds), dim3(256), lds, stream, a);
    return launched();
}
// `a`, whose operands, sizes, outputs and segs / results are set (rows aligned and near), gets the rest by `plan`.
inline int place_tiles(Args &a, const Plan &plan, void *workspace, int xcds) {
    a.tiles_m = plan.tiles_m; a.tiles_n = plan.tiles_n; a.ktiles = plan.ktiles; a.splits = plan.splits;
    if (plan.splits > 1 && !workspace) return ALCS_E_INVALID_ARG;
    a.partial = plan.splits > 1 ? (float *)workspace : nullptr;
    const long long total = (long long)a.tiles_m * a.tiles_n * a.results * a.splits;
    if (total >= (1 << 24) - 64) return ALCS_E_UNSUPPORTED;  // a launch has less than 2^32 threads
    a.total = (unsigned)total;
    a.xcds = (unsigned)xcds;
    a.per_xcd = (unsigned)((total + xcds - 1) / xcds);
    return ALCS_OK;
}
template <class T, bool GATED> int launch_join(const Args &a, hipStream_t stream) {
    if (a.splits == 1) return ALCS_OK;
    const long long quads = (long long)(GATED ? 1 : a.results) * a.M * ((a.N + 3) / 4);
    hipLaunchKernelGGL((k_join<T, GATED>), dim3((unsigned)((quads + 255) / 256)), dim3(256), 0, stream, a);
    return launched();
}
template <int E, class T, bool AK, bool BK, bool GATED>
int launch_tiles(Args a, const Plan &plan, void *workspace, int cus, int xcds, hipStream_t stream) {
    int rc = place_tiles(a, plan, workspace, xcds);
    if (rc != ALCS_OK) return rc;
    if (deep_tiles(E, BK, plan, a.results, cus)) {
        if constexpr (E != kF32 && !BK) rc = launch_mid<E, T, 128, 4, AK, BK, GATED>(a, stream);
    } else if (plan.kind == k128) {
        rc = launch_mid<E, T, 128, stages_of(128), AK, BK, GATED>(a, stream);
    } else if (plan.kind == k64) {
        rc = launch_mid<E, T, 64, stages_of(64), AK, BK, GATED>(a, stream);
    } else {
        if constexpr (E != kF32) rc = launch_big<E, T, AK, BK, GATED>(a, cus, stream);
    }
    return rc == ALCS_OK ? launch_join<T, GATED>(a, stream) : rc;
}

template <int E, class T, int BMX, int BMW> int launch_pair_as(const Args &x, const Args &w, const BiasArgs &b, bool x_first, hipStream_t stream) {
    constexpr int lds = std::max(stages_of(BMX) * Feed<E, BMX, 128, false, true, false>::kBuf, stages_of(BMW) * Feed<E, BMW, 128, true, true, false>::kBuf);
    static_assert(lds <= 80 * 1024, "two workgroups on a compute unit");
    auto kern = k_pair<E, T, BMX, BMW>;
    const int rc = allow_lds((const void *)kern, lds);
    if (rc != ALCS_OK) return rc;
    const unsigned nx = x.per_xcd * x.xcds, nw = w.per_xcd * w.xcds;
    hipLaunchKernelGGL(kern, dim3(nx + nw + b.blocks), dim3(256), lds, stream, x, w, b, nx, nw, (int)x_first);
    return launched();
}
template <int E, class T> int launch_pair(Args x, Args w, const BiasArgs &b, const Shape &sx, const Shape &sw, const Plans &p, char *workspace, int xcds, hipStream_t stream) {
    int rc = place_tiles(x, p.x, workspace, xcds);
    if (rc == ALCS_OK) rc = place_tiles(w, p.w, workspace + whole256(p.x.workspace), xcds);
    if (rc != ALCS_OK) return rc;
    const bool first = depth_of(sx, p.x) * cost_of(sx, p.x.kind).two >= depth_of(sw, p.w) * cost_of(sw, p.w.kind).two;
    if (p.x.kind == k128) rc = p.w.kind == k128 ? launch_pair_as<E, T, 128, 128>(x, w, b, first, stream) : launch_pair_as<E, T, 128, 64>(x, w, b, first, stream);
    else rc = p.w.kind == k128 ? launch_pair_as<E, T, 64, 128>(x, w, b, first, stream) : launch_pair_as<E, T, 64, 64>(x, w, b, first, stream);
    if (rc == ALCS_OK) rc = launch_join<T, false>(x, stream);
    return rc == ALCS_OK ? launch_join<T, false>(w, stream) : rc;
}
template <int E, class T, bool GATED, bool ALIGNED> int launch_few_as(const Args &a, hipStream_t stream) {
    const int pieces = (a.KA + 16 * per16(E) - 1) / (16 * per16(E)), W = std::max(1, std::min(8, pieces));
    const int MF = a.M <= 16 ? 1 : a.M <= 32 ? 2 : 4, lds = W * (GATED ? 2 : 1) * MF * 1024;
    auto kern = MF == 1 ? k_few<E, T, 1, GATED, ALIGNED> : MF == 2 ? k_few<E, T, 2, GATED, ALIGNED> : k_few<E, T, 4, GATED, ALIGNED>;
    const int rc = allow_lds((const void *)kern, lds);
    if (rc != ALCS_OK) return rc;
    const long long blocks = up(a.N, 16) * up(a.M, 16 * MF);
    if (blocks >= 1 << 23) return ALCS_E_UNSUPPORTED;  // a launch has less than 2^32 threads
    hipLaunchKernelGGL(kern, dim3((unsigned)blocks), dim3(W * 64), lds, stream, a);
    return launched();
}
template <int E, class T, bool GATED> int launch_few(const Args &a, bool aligned, hipStream_t stream) {
    if constexpr (E == kMX4) return launch_few_as<E, T, GATED, true>(a, stream);
    else return aligned ? launch_few_as<E, T, GATED, true>(a, stream) : launch_few_as<E, T, GATED, false>(a, stream);
}

}  // namespace tile
}  // namespace alcs
