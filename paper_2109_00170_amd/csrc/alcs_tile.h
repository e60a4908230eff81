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
// lane fetches.  Two K tiles are in LDS: while one is multiplied, the other is on its way.
//
// Layouts.  "K contiguous" (rows of A and B as a linear layer has them): [row][128 bytes], the 16-byte
// piece c of row r at position c ^ (r & 7).  "K strided" (the operands of a gradient, whose sum runs over
// rows): [k][row], read transposed - by the LDS load that transposes 16-bit values, float by float for
// float32 -, in units of 16 rows whose positions are exchanged among the k that one load reads together.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "alcs_internal.h"

namespace alcs {
namespace tile {

enum Elem { kF32 = 0, kBF16 = 1, kF16 = 2, kMX4 = 3 };
constexpr int bytes_of(int E) { return E == kF32 ? 4 : 2; }                  // not for kMX4
constexpr int per16(int E) { return E == kF32 ? 4 : E == kMX4 ? 32 : 8; }    // elements in 16 bytes
constexpr int kTileBytes = 128;                                              // of K, per row

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
// for results of 16 bits the hardware's exp2 and reciprocal (relative error about 2^-22) are far below the rounding.
template <bool EXACT> __device__ inline float sigmoid(float g) {
    if (EXACT) return 1.0f / (1.0f + expf(-g));
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g * -1.44269504f));
}
constexpr float kGeluA = 0.7978845608f, kGeluB = 0.044715f;  // sqrt(2/pi)
template <bool EXACT> __device__ inline float gate_value(int gate, float g) {
    switch (gate) {
        case ALCS_GATE_RELU: return g < 0.0f ? 0.0f : g;
        case ALCS_GATE_SILU: return g * sigmoid<EXACT>(g);
        case ALCS_GATE_GELU: return 0.5f * g * (1.0f + erff(g * 0.70710678f));
        // 0.5 (1 + tanh z) = sigmoid(2 z)
        case ALCS_GATE_GELU_TANH: return g * sigmoid<EXACT>(2.0f * kGeluA * (g + kGeluB * g * g * g));
        case ALCS_GATE_SIGMOID: return sigmoid<EXACT>(g);
        default: return g;
    }
}
// value and derivative
template <bool EXACT> __device__ inline void gate_both(int gate, float g, float &v, float &d) {
    switch (gate) {
        case ALCS_GATE_RELU: v = g < 0.0f ? 0.0f : g; d = g > 0.0f ? 1.0f : 0.0f; break;
        case ALCS_GATE_SILU: { const float s = sigmoid<EXACT>(g); v = g * s; d = s * (1.0f + g * (1.0f - s)); break; }
        case ALCS_GATE_GELU: {
            const float c = 0.5f * (1.0f + erff(g * 0.70710678f));
            v = g * c;
            d = c + g * 0.3989422804f * expf(-0.5f * g * g);
            break;
        }
        case ALCS_GATE_GELU_TANH: {
            const float s = sigmoid<EXACT>(2.0f * kGeluA * (g + kGeluB * g * g * g));
            v = g * s;
            d = s + g * s * (1.0f - s) * 2.0f * kGeluA * (1.0f + 3.0f * kGeluB * g * g);
            break;
        }
        case ALCS_GATE_SIGMOID: { const float s = sigmoid<EXACT>(g); v = s; d = s * (1.0f - s); break; }
        default: v = g; d = 1.0f;
    }
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
    int rows;              // K strided: elements of a k that may be read (whole pieces where the operand is aligned)
};
struct Args {
    Operand A[2], B[2];  // of the K segments (segs = 2), of the two results (results = 2), or gate and up (B)
    int M, N;            // rows and columns of the result; for a gated product N columns of each projection
    int KA, KB;          // elements of K that A and B hold (A may be padded with zeros beyond B's)
    int segs, results;
    int tiles_m, tiles_n, splits, ktiles;  // ktiles: K tiles of a segment
    unsigned total, per_xcd, xcds;
    float *partial;      // splits > 1: [split][plane][M][N] sums
    const float *bias[2];
    void *out[2];        // the result(s); gated: H
    void *pre[2];        // gated: G and U where the caller keeps them, or null
    long long ldo;       // elements from one row of out (and pre) to the next
    int act;             // alcs_activation, or alcs_gate for a gated product
    int vec;             // rows of out and pre may be written four elements at a time
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

typedef __attribute__((address_space(3))) char lds_char;
__device__ inline unsigned lds_offset(const char *p) { return (unsigned)(uintptr_t)(lds_char *)(char *)p; }

// ------------------------------------------------------------------------------ one operand's tile

// R rows (of A, or of B: both projections' for a gated product) and 128 bytes of K, brought in by W wavefronts.
template <int E, int R, int W, bool KSTRIDED, bool ALIGNED> struct Stage {
    static constexpr int kElems = per16(E), kK = 8 * kElems;
    static constexpr int kBytes = R * kTileBytes, kLoads = kBytes / 1024 / W;
    static constexpr int kScaleLoads = E == kMX4 ? R * 8 / 256 / W : 0;
    static_assert(kBytes % (1024 * W) == 0 && (E != kMX4 || R * 8 % (256 * W) == 0), "whole loads per wavefront");
    const char *ptr[kLoads];
    const char *sptr[kScaleLoads ? kScaleLoads : 1];
    int k_of[kLoads];   // first k (K contiguous: of the piece; K strided: the row) inside the tile
    int left[kLoads];   // K strided: elements of the piece inside the operand
    v4i held[ALIGNED ? 1 : kLoads];

    // where lane `lane`'s piece of load i lies: row of the tile (K contiguous) or k and first row (K strided)
    static __device__ void place(int i, int wave, int lane, int &row, int &k) {
        const int o = (wave * kLoads + i) * 1024 + lane * 16;
        if (!KSTRIDED) {
            row = o / kTileBytes;
            k = (((o / 16) & 7) ^ (row & 7)) * kElems;
        } else {
            constexpr int RB = R * (E == kF32 ? 4 : 2);
            k = o / RB;
            const int piece = (o % RB) / 16;
            if (E == kF32) row = ((piece >> 2) ^ ((k >> 2) & 3)) * 16 + (piece & 3) * 4;
            else row = ((piece >> 1) ^ ((k & 3) | ((k >> 1) & 4))) * 16 + (piece & 1) * 8;
        }
    }
    // K contiguous: row_of(row) = where tile row `row` starts (of a row that exists)
    template <class F> __device__ void start_rows(int wave, int lane, int k0, F row_of) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            int row;
            place(i, wave, lane, row, k_of[i]);
            ptr[i] = row_of(row) + (long long)(k0 + k_of[i]) / kElems * 16;
        }
    }
    // K strided: tile row 0 is element `first` of every k
    __device__ void start_columns(int wave, int lane, int k0, const char *p, long long pitch, int first, int rows) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            int row;
            place(i, wave, lane, row, k_of[i]);
            const int r = first + row, l = rows - r;
            left[i] = l < 0 ? 0 : l > kElems ? kElems : l;
            // aligned operands have whole pieces: one beyond them reads the last, for columns that nobody stores
            ptr[i] = p + (k0 + k_of[i]) * pitch + (long long)(ALIGNED && l < kElems ? rows - kElems : r) * bytes_of(E);
        }
    }
    // row_of(row) = where the scales of tile row `row` start; the tile's scales lie in LDS as dwords (four blocks),
    // [64 rows][row & 15][half of the tile][16 rows], so that a lane reads those of four fragments at once
    template <class F> __device__ void start_scales(int wave, int lane, int k0, F row_of) {
#pragma unroll
        for (int i = 0; i < kScaleLoads; ++i) {
            const int d = (wave * kScaleLoads + i) * 64 + lane;
            sptr[i] = row_of(((d >> 7) * 4 + (d & 3)) * 16 + ((d >> 3) & 15)) + k0 / 32 + ((d >> 2) & 1) * 4;
        }
    }
    // the loads of the K tile that starts at k0 (of K) into the LDS region at `lds`; `step` bytes to the next one
    __device__ void issue(int k0, int K, unsigned lds, unsigned slds, int wave, int lane, long long step) {
        const bool whole = k0 + kK <= K;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            if (ALIGNED) {
                const char *g = ptr[i];
                if (!whole && k0 + k_of[i] >= K) g = (const char *)g_zeros;
                lds_load16(g, lds + (wave * kLoads + i) * 1024);
            } else {
                held[i] = fetch(i, k0, K);
            }
            ptr[i] += step;
        }
        if (E == kMX4) {
#pragma unroll
            for (int i = 0; i < kScaleLoads; ++i) {
                const char *g = sptr[i];
                if (!whole && k0 + ((lane >> 2) & 1) * 128 >= K) g = (const char *)g_zeros;
                lds_load4(g, slds + (wave * kScaleLoads + i) * 256);
                sptr[i] += 8;
            }
        }
    }
    // unaligned operands: through registers, a piece that is not whole element by element
    __device__ v4i fetch(int i, int k0, int K) const {
        typedef typename TypeOf<E>::type T;
        v4i v = {0, 0, 0, 0};
        int n;
        if (KSTRIDED) n = k0 + k_of[i] < K ? left[i] : 0;
        else n = K - (k0 + k_of[i]) < 0 ? 0 : K - (k0 + k_of[i]) > kElems ? kElems : K - (k0 + k_of[i]);
        if (n == kElems) {
            __builtin_memcpy(&v, ptr[i], 16);
        } else {
            T e[kElems] = {};
#pragma unroll
            for (int j = 0; j < kElems; ++j)
                if (j < n) __builtin_memcpy(&e[j], ptr[i] + j * sizeof(T), sizeof(T));
            __builtin_memcpy(&v, e, 16);
        }
        return v;
    }
    __device__ void put(char *lds, int wave, int lane) const {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) *(v4i *)(lds + (wave * kLoads + i) * 1024 + lane * 16) = held[i];
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
            const int piece = E == kMX4 ? 2 * q + s : 4 * s + q;
            return *(const v4i *)(lds + (first + f * 16 + r) * kTileBytes + ((piece ^ (r & 7)) << 4));
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
        const char *p = lds + k * RB + ((u ^ ((r >> 2) | ((q & 1) << 2))) << 5) + (r & 3) * 8;
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

// ------------------------------------------------------------------------------ what follows the sum

template <class T> __device__ inline void store4(T *p, const float v[4], int n, int vec) {
    if (vec && n >= 4) {
        struct alignas(sizeof(T) * 4) Four { T e[4]; } f;
#pragma unroll
        for (int i = 0; i < 4; ++i) f.e[i] = (T)v[i];
        *(Four *)p = f;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) p[i] = (T)v[i];
    }
}
// four neighbours of a row: bias, activation, rounding (once, to the result's type)
template <class T> __device__ inline void finish_plain(const Args &a, int result, long long m, int n, v4f c) {
    const int left = a.N - n;
    if (left <= 0) return;
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = activate(a.act, c[i] + (a.bias[0] && i < left ? a.bias[0][n + i] : 0.0f));
    store4((T *)a.out[result] + m * a.ldo + n, v, left, a.vec);
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
    store4((T *)a.out[0] + at, h, left, a.vec);
    if (a.pre[0]) {
        store4((T *)a.pre[0] + at, gg, left, a.vec);
        store4((T *)a.pre[1] + at, uu, left, a.vec);
    }
}

// ------------------------------------------------------------------------------ the kernel

// The tile of a workgroup: workgroups are dealt round-robin to the XCDs, so numbers are exchanged such that
// an XCD works on neighbouring tiles, columns of up to 8 tiles of rows at a time, and shares their operands in its L2.
__device__ inline bool tile_of(const Args &a, int &m, int &n, int &z) {
    const unsigned id = (blockIdx.x % a.xcds) * a.per_xcd + blockIdx.x / a.xcds;
    if (id >= a.total) return false;
    const unsigned per = (unsigned)a.tiles_m * a.tiles_n;
    z = (int)(id / per);
    const unsigned t = id % per, strip = t / (8u * a.tiles_n), in = t % (8u * a.tiles_n);
    const unsigned first = strip * 8, rows = min(8u, (unsigned)a.tiles_m - first);
    m = (int)(first + in % rows);
    n = (int)(in / rows);
    return true;
}

template <int E, class T, int BM, int BN, int WM, int WN, bool AK, bool BK, bool GATED, bool ALIGNED>
__global__ __launch_bounds__(WM *WN * 64, 2) void k_tile(const Args a) {
    constexpr int W = WM * WN, FM = BM / WM / 16, FN = BN / WN / 16;
    constexpr int kA = BM * kTileBytes, kB = BN * kTileBytes, kS = E == kMX4 ? (BM + BN) * 8 : 0;
    constexpr int kBuf = kA + kB + kS, kK = 8 * per16(E);
    extern __shared__ __align__(16) char lds[];
    int tm, tn, z;
    if (!tile_of(a, tm, tn, z)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const int m0 = tm * BM, n0 = tn * (GATED ? BN / 2 : BN);
    const int result = a.results == 2 ? z & 1 : 0, split = a.results == 2 ? z >> 1 : z;
    // this split's K tiles, over all segments
    const int all = a.ktiles * a.segs;
    const int from = (int)((long long)all * split / a.splits), to = (int)((long long)all * (split + 1) / a.splits);

    v4f acc[FM][FN] = {};
    Stage<E, BM, W, AK, ALIGNED> sa;
    Stage<E, BN, W, BK, ALIGNED> sb;
    int seg = -1;
    long long stepA = 0, stepB = 0;
    auto issue = [&](int t, int buf) {
        const int s = t / a.ktiles, k0 = (t - s * a.ktiles) * kK;
        if (s != seg) {  // the first tile, or the first of the next segment
            seg = s;
            const bool second = a.segs == 2 ? s == 1 : result == 1;
            const char *pa = second ? a.A[1].p : a.A[0].p, *pb = a.segs == 2 && s == 1 ? a.B[1].p : a.B[0].p;
            const long long pitchA = second ? a.A[1].pitch : a.A[0].pitch;
            const long long pitchB = a.segs == 2 && s == 1 ? a.B[1].pitch : a.B[0].pitch;
            stepA = AK ? pitchA * kK : kTileBytes;
            stepB = BK ? pitchB * kK : kTileBytes;
            if (AK) sa.start_columns(wave, lane, k0, pa, pitchA, m0, a.A[0].rows);
            else sa.start_rows(wave, lane, k0, [&](int row) { return pa + min(m0 + row, a.M - 1) * pitchA; });
            if (BK) sb.start_columns(wave, lane, k0, pb, pitchB, n0, a.B[0].rows);
            else if (GATED) sb.start_rows(wave, lane, k0, [&](int row) {
                // a wavefront's columns: half of them of the gate, half of the other projection
                constexpr int half = BN / WN / 2;
                const int w = row / (2 * half), j = row % (2 * half), n = min(n0 + w * half + j % half, a.N - 1);
                return j < half ? a.B[0].p + n * a.B[0].pitch : a.B[1].p + n * a.B[1].pitch;
            });
            else sb.start_rows(wave, lane, k0, [&](int row) { return pb + min(n0 + row, a.N - 1) * pitchB; });
            if (E == kMX4) {
                sa.start_scales(wave, lane, k0, [&](int row) {
                    return (const char *)a.A[0].scales + min(m0 + row, a.M - 1) * (pitchA / 16);
                });
                sb.start_scales(wave, lane, k0, [&](int row) {
                    return (const char *)a.B[0].scales + min(n0 + row, a.N - 1) * (pitchB / 16);
                });
            }
        }
        const unsigned at = lds_offset(lds) + buf * kBuf;
        sa.issue(k0, a.KA, at, at + kA + kB, wave, lane, stepA);
        sb.issue(k0, a.KB, at + kA, at + kA + kB + BM * 8, wave, lane, stepB);
    };
    const Reader<E, BM, AK> ra(wm * FM * 16, lane);
    const Reader<E, BN, BK> rb(wn * FN * 16, lane);

    if (from < to) issue(from, 0);
    for (int t = from; t < to; ++t) {
        const int buf = (t - from) & 1;
        char *here = lds + buf * kBuf;
        if (!ALIGNED) {
            sa.put(here, wave, lane);
            sb.put(here + kA, wave, lane);
        }
        wait_loads();
        __syncthreads();  // this tile is there, and nobody reads the other buffer any more
        if (t + 1 < to) issue(t + 1, buf ^ 1);
        int sca[FM], scb[FN];
        if (E == kMX4) {
            // a lane's two blocks of a tile are 2q and 2q + 1: a dword of four fragments' at a time, shifted so
            // that step s takes byte s
            const int at = ((lane & 15) * 2 + (lane >> 5)) * 16, shift = (lane & 16);
#pragma unroll
            for (int f = 0; f < FM; f += 4) {
                const v4i v = *(const v4i *)(here + kA + kB + (wm * FM + f) * 128 + at);
#pragma unroll
                for (int j = 0; j < 4; ++j) sca[f + j] = (unsigned)v[j] >> shift;
            }
#pragma unroll
            for (int f = 0; f < FN; f += 4) {
                const v4i v = *(const v4i *)(here + kA + kB + BM * 8 + (wn * FN + f) * 128 + at);
#pragma unroll
                for (int j = 0; j < 4; ++j) scb[f + j] = (unsigned)v[j] >> shift;
            }
        }
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            v4i fa[FM], fb[FN];
#pragma unroll
            for (int f = 0; f < FN; ++f) fb[f] = rb.get(here + kA, f, s);
#pragma unroll
            for (int f = 0; f < FM; ++f) fa[f] = ra.get(here, f, s);
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j)
                    acc[i][j] = multiply<E>(fb[j], fa[i], acc[i][j], s, E == kMX4 ? scb[j] : 0, E == kMX4 ? sca[i] : 0);
        }
    }

    const int r = lane & 15, q = lane >> 4;
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        const int m = m0 + (wm * FM + i) * 16 + r;
        if (m >= a.M) continue;
        if (GATED) {
#pragma unroll
            for (int j = 0; j < FN / 2; ++j) {
                const int n = n0 + (wn * FN / 2 + j) * 16 + q * 4;
                if (a.partial) {
                    float *p = a.partial + ((long long)split * 2 * a.M + m) * a.N + n;
                    const float g[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
                    const v4f uv = acc[i][j + FN / 2];
                    const float u[4] = {uv[0], uv[1], uv[2], uv[3]};
                    if (a.N > n) {
                        store4(p, g, a.N - n, a.N % 4 == 0);
                        store4(p + (long long)a.M * a.N, u, a.N - n, a.N % 4 == 0);
                    }
                } else {
                    finish_gated<T>(a, m, n, acc[i][j], acc[i][j + FN / 2]);
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                const int n = n0 + (wn * FN + j) * 16 + q * 4;
                if (a.partial) {
                    const float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
                    if (a.N > n)
                        store4(a.partial + (((long long)split * a.results + result) * a.M + m) * a.N + n, v, a.N - n, a.N % 4 == 0);
                } else {
                    finish_plain<T>(a, result, m, n, acc[i][j]);
                }
            }
        }
    }
}

// The sums of a split K, added in the order of the splits; a thread has four neighbours of a row.
template <class T, bool GATED> __global__ __launch_bounds__(256) void k_join(const Args a) {
    const int quads = (a.N + 3) / 4;
    const long long at = (long long)blockIdx.x * 256 + threadIdx.x;
    const int planes = GATED ? 1 : a.results;
    if (at >= (long long)planes * a.M * quads) return;
    const int n = (int)(at % quads) * 4;
    const long long row = at / quads;  // plane * M + m
    const long long plane = (long long)(GATED ? 2 : a.results) * a.M * a.N;
    const int left = min(4, a.N - n);
    v4f s[2] = {};
    for (int k = 0; k < a.splits; ++k)
#pragma unroll
        for (int h = 0; h < (GATED ? 2 : 1); ++h) {
            const float *p = a.partial + k * plane + (row + (long long)h * a.M) * a.N + n;
            if (a.N % 4 == 0) s[h] += *(const v4f *)p;
            else
                for (int i = 0; i < left; ++i) s[h][i] += p[i];
        }
    if (GATED) finish_gated<T>(a, row, n, s[0], s[1]);
    else finish_plain<T>(a, (int)(row / a.M), row % a.M, n, s[0]);
}

// ------------------------------------------------------------------------------ few rows

// Up to 16 * MF rows of A (a token, a few requests): the weights are read once and the product is bound by
// their bytes, so nothing is staged.  A workgroup has 16 columns (of both projections where GATED); its wavefronts
// share out K in pieces of 256 bytes a row, read their fragments straight from memory, four steps ahead of
// the multiply, and add their sums through LDS in a fixed order.  Rows of A beyond M read the last row.
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
    const int r = lane & 15, q = lane >> 4, n0 = blockIdx.x * 16;
    const int n = min(n0 + r, a.N - 1);
    const char *w[P];
#pragma unroll
    for (int p = 0; p < P; ++p) w[p] = a.B[p].p + n * a.B[p].pitch;
    const char *x[MF];
    const char *xs[MF], *ws = nullptr;
#pragma unroll
    for (int f = 0; f < MF; ++f) {
        const int m = min(f * 16 + r, a.M - 1);
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
        const int m = f * 16 + r;
        if (m < a.M) {
            if (GATED) finish_gated<T>(a, m, n0 + q * 4, s[0], s[P - 1]);
            else finish_plain<T>(a, 0, m, n0 + q * 4, s[0]);
        }
    }
}

// ------------------------------------------------------------------------------ launches

struct Plan {
    bool big;    // 256 x 256 tiles, eight wavefronts; else 128 x 128, four
    int tiles_m, tiles_n, ktiles, splits;
    long long workspace;  // bytes of sums that a split needs
};
// M rows and N columns (of each projection where gated), `results` of them, K elements in each of `segs` segments.
inline Plan plan_tiles(int E, bool aligned, bool gated, long long M, long long N, long long K, int segs, int results, int cus) {
    auto up = [](long long a, long long b) { return (a + b - 1) / b; };
    Plan p{};
    p.ktiles = (int)up(K, 8 * per16(E));
    p.big = aligned && E != kF32 && up(M, 256) * up(N, gated ? 128 : 256) * results >= cus / 2;
    const int side = p.big ? 256 : 128;
    p.tiles_m = (int)up(M, side);
    p.tiles_n = (int)up(N, gated ? side / 2 : side);
    p.splits = 1;
    const long long tiles = (long long)p.tiles_m * p.tiles_n * results, all = (long long)p.ktiles * segs;
    // two of the small tiles run on a compute unit; a part of K is at least four tiles of it
    if (!p.big && tiles < cus) p.splits = (int)std::max(1LL, std::min({2LL * cus / tiles, all / 4, 16LL}));
    p.workspace = p.splits > 1 ? (long long)p.splits * (gated ? 2 : results) * M * N * 4 : 0;
    return p;
}
inline long long workspace_of(int E, bool gated, long long M, long long N, long long K, int segs, int results, int cus) {
    const long long a = plan_tiles(E, true, gated, M, N, K, segs, results, cus).workspace;
    return E == kMX4 ? a : std::max(a, plan_tiles(E, false, gated, M, N, K, segs, results, cus).workspace);
}
inline int launched() {
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return ALCS_OK;
    set_hip_error((int)e);
    return ALCS_E_HIP;
}

template <int E, class T, int BM, int BN, int WM, int WN, bool AK, bool BK, bool GATED, bool ALIGNED>
int launch_one(Args &a, hipStream_t stream) {
    constexpr int lds = 2 * ((BM + BN) * kTileBytes + (E == kMX4 ? (BM + BN) * 8 : 0));
    auto kern = k_tile<E, T, BM, BN, WM, WN, AK, BK, GATED, ALIGNED>;
    const int rc = allow_lds((const void *)kern, lds);
    if (rc != ALCS_OK) return rc;
    hipLaunchKernelGGL(kern, dim3(a.per_xcd * a.xcds), dim3(WM * WN * 64), lds, stream, a);
    return launched();
}
// The product that `a` describes (operands, sizes, outputs and segs / results set), tiles by `plan`.
template <int E, class T, bool AK, bool BK, bool GATED>
int launch_tiles(Args a, const Plan &plan, bool aligned, void *workspace, int cus, int xcds, hipStream_t stream) {
    a.tiles_m = plan.tiles_m; a.tiles_n = plan.tiles_n; a.ktiles = plan.ktiles; a.splits = plan.splits;
    a.partial = plan.splits > 1 ? (float *)workspace : nullptr;
    const long long total = (long long)a.tiles_m * a.tiles_n * a.results * a.splits;
    if (total > INT32_MAX - 64) return ALCS_E_UNSUPPORTED;
    a.total = (unsigned)total;
    a.xcds = (unsigned)xcds;
    a.per_xcd = (unsigned)((total + xcds - 1) / xcds);
    int rc;
    if constexpr (E == kMX4) {
        rc = plan.big ? launch_one<E, T, 256, 256, 2, 4, AK, BK, GATED, true>(a, stream)
                      : launch_one<E, T, 128, 128, 2, 2, AK, BK, GATED, true>(a, stream);
    } else if constexpr (E == kF32) {
        rc = aligned ? launch_one<E, T, 128, 128, 2, 2, AK, BK, GATED, true>(a, stream)
                     : launch_one<E, T, 128, 128, 2, 2, AK, BK, GATED, false>(a, stream);
    } else {
        rc = !aligned ? launch_one<E, T, 128, 128, 2, 2, AK, BK, GATED, false>(a, stream)
             : plan.big ? launch_one<E, T, 256, 256, 2, 4, AK, BK, GATED, true>(a, stream)
                        : launch_one<E, T, 128, 128, 2, 2, AK, BK, GATED, true>(a, stream);
    }
    if (rc != ALCS_OK || a.splits == 1) return rc;
    const long long quads = (long long)(GATED ? 1 : a.results) * a.M * ((a.N + 3) / 4);
    hipLaunchKernelGGL((k_join<T, GATED>), dim3((unsigned)((quads + 255) / 256)), dim3(256), 0, stream, a);
    return launched();
}
constexpr int kFewRows = 64;
template <int E, class T, bool GATED, bool ALIGNED> int launch_few_as(const Args &a, hipStream_t stream) {
    const int pieces = (a.KA + 16 * per16(E) - 1) / (16 * per16(E)), W = std::max(1, std::min(8, pieces));
    const int MF = a.M <= 16 ? 1 : a.M <= 32 ? 2 : 4, lds = W * (GATED ? 2 : 1) * MF * 1024;
    auto kern = MF == 1 ? k_few<E, T, 1, GATED, ALIGNED> : MF == 2 ? k_few<E, T, 2, GATED, ALIGNED> : k_few<E, T, 4, GATED, ALIGNED>;
    const int rc = allow_lds((const void *)kern, lds);
    if (rc != ALCS_OK) return rc;
    hipLaunchKernelGGL(kern, dim3((unsigned)((a.N + 15) / 16)), dim3(W * 64), lds, stream, a);
    return launched();
}
template <int E, class T, bool GATED> int launch_few(const Args &a, bool aligned, hipStream_t stream) {
    if constexpr (E == kMX4) return launch_few_as<E, T, GATED, true>(a, stream);
    else return aligned ? launch_few_as<E, T, GATED, true>(a, stream) : launch_few_as<E, T, GATED, false>(a, stream);
}

}  // namespace tile
}  // namespace alcs
