// Microscaled 4-bit storage (alcs.h): to it, back from it, and the product of two matrices held in it.
#include "alcs_tile.h"

namespace alcs {
namespace tile {

// ------------------------------------------------------------------------------ to storage and back

// A thread has eight neighbouring columns: 16 or 32 bytes in, four bytes of codes out.  Four threads share a
// block and exchange its largest magnitude (compared as bit patterns, so that a NaN is larger than anything),
// sixteen a dword of scales.  The block's exponent field less two is the scale byte (never below 0: elements of
// up to 2^-125 are held in units of 2^-127), and the conversion instruction divides by it, rounds to nearest
// even and saturates.  Bound by memory.
template <class T> __device__ inline void load8(const T *p, int n, float v[8]) {
    if (n >= 8) {
        T e[8];
        __builtin_memcpy(e, p, sizeof(e));
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = to_float(e[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? to_float(p[i]) : 0.0f;
    }
}

template <class T> __global__ __launch_bounds__(256) void k_mx4_quantize(const T *X, long long ldx, long long rows, int cols,
                                                                        int eights, uint32_t *codes, uint32_t *scales) {
    const unsigned at = blockIdx.x * 256 + threadIdx.x;  // eights (per row) is a multiple of 16
    if (at >= rows * eights) return;                     // whole groups of 16 threads leave
    const unsigned row = at / (unsigned)eights;
    const int c = (int)(at % (unsigned)eights) * 8;
    float v[8];
    load8(X + row * ldx + c, cols - c, v);
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
    top = max(top, (uint32_t)__shfl_xor((int)top, 1));
    top = max(top, (uint32_t)__shfl_xor((int)top, 2));
    const bool bad = top >= 0x7f800000u;
    const uint32_t field = top >> 23, scale = field > 2 ? field - 2 : 0;
    const float unit = __uint_as_float(scale ? scale << 23 : 1u << 22);
    uint32_t code = 0;
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[0], v[1], unit, 0);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[2], v[3], unit, 1);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[4], v[5], unit, 2);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[6], v[7], unit, 3);
    codes[at] = bad ? 0u : code;
    // the four blocks of sixteen threads
    uint32_t byte = (bad ? 255u : scale) << ((threadIdx.x >> 2 & 3) * 8);
    byte |= (uint32_t)__shfl_xor((int)byte, 4);
    byte |= (uint32_t)__shfl_xor((int)byte, 8);
    if ((threadIdx.x & 15) == 0) scales[at / 16] = byte;
}

// A thread has 16 bytes of the result (4 or 8 columns), so that a wavefront's stores are one run.  Bound by the stores.
template <class T> __global__ __launch_bounds__(256) void k_mx4_dequantize(const uint8_t *codes, const uint8_t *scales, long long rows,
                                                                          int cols, int pieces, T *Y) {
    constexpr int kN = 16 / sizeof(T);  // pieces: of a row's stored columns
    const unsigned at = blockIdx.x * 256 + threadIdx.x;
    if (at >= rows * pieces) return;
    const unsigned row = at / (unsigned)pieces;
    const int c = (int)(at % (unsigned)pieces) * kN, n = cols - c;
    if (n <= 0) return;
    const uint32_t code = kN == 8 ? ((const uint32_t *)codes)[at] : ((const uint16_t *)codes)[at], scale = scales[at / (32 / kN)];
    const float unit = __uint_as_float(scale ? scale << 23 : 1u << 22), nan = __uint_as_float(0x7fc00000u);
    typedef float v2f __attribute__((ext_vector_type(2)));
    v2f w[4];
    w[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, unit, 0);
    w[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, unit, 1);
    if (kN == 8) {
        w[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, unit, 2);
        w[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, unit, 3);
    }
    T out[kN];
#pragma unroll
    for (int i = 0; i < kN; ++i) out[i] = (T)(scale == 255 ? nan : w[i / 2][i % 2]);
    T *p = Y + (long long)row * cols + c;
    if (n >= kN) {
        v4i v;
        __builtin_memcpy(&v, out, 16);
        __builtin_memcpy(p, &v, 16);
    } else {
#pragma unroll
        for (int i = 0; i < kN; ++i)
            if (i < n) p[i] = out[i];
    }
}

inline int check_stored(const void *codes, const void *scales) {
    return codes && scales && (uintptr_t)codes % 16 == 0 && (uintptr_t)scales % 4 == 0 ? ALCS_OK : ALCS_E_INVALID_ARG;
}
constexpr int kMaxSize = 1 << 26;

template <class T> int linear_as(const Args &a, void *workspace, long long workspace_bytes, int cus, int xcds, hipStream_t stream) {
    if (few_rows(kMX4, a.M, a.N, a.KA, false, cus)) return launch_few<kMX4, T, false>(a, true, stream);
    const Plan p = plan_tiles(linear_shape(a.M, a.N, a.KA), workspace ? workspace_bytes : 0, cus);
    return launch_tiles<kMX4, T, false, false, false>(a, p, workspace, cus, xcds, stream);
}

}  // namespace tile
}  // namespace alcs

using namespace alcs;
using namespace alcs::tile;

extern "C" int alcs_mx4_quantize(const void *X_dev, long long ldx, long long rows, int cols, int dtype, uint8_t *codes_dev,
                                 uint8_t *scales_dev, void *stream) {
    if (rows < 0 || cols <= 0 || ldx < 0 || dtype < ALCS_F32 || dtype > ALCS_F16) return ALCS_E_INVALID_ARG;
    if (cols > tile::kMaxSize) return ALCS_E_UNSUPPORTED;
    if (rows == 0) return ALCS_OK;
    if (!X_dev || check_stored(codes_dev, scales_dev) != ALCS_OK) return ALCS_E_INVALID_ARG;
    const int eights = (cols + 127) / 128 * 16;
    if (rows > ((1LL << 32) - 512) / eights) return ALCS_E_UNSUPPORTED;  // a launch has less than 2^32 threads
    const dim3 grid((unsigned)((rows * eights + 255) / 256));
    uint32_t *c = (uint32_t *)codes_dev, *s = (uint32_t *)scales_dev;
    const hipStream_t st = (hipStream_t)stream;
    if (dtype == ALCS_F32)
        hipLaunchKernelGGL(k_mx4_quantize<float>, grid, dim3(256), 0, st, (const float *)X_dev, ldx, rows, cols, eights, c, s);
    else if (dtype == ALCS_BF16)
        hipLaunchKernelGGL(k_mx4_quantize<__bf16>, grid, dim3(256), 0, st, (const __bf16 *)X_dev, ldx, rows, cols, eights, c, s);
    else
        hipLaunchKernelGGL(k_mx4_quantize<_Float16>, grid, dim3(256), 0, st, (const _Float16 *)X_dev, ldx, rows, cols, eights, c, s);
    return launched();
}

extern "C" int alcs_mx4_dequantize(const uint8_t *codes_dev, const uint8_t *scales_dev, long long rows, int cols, int dtype,
                                   void *Y_dev, void *stream) {
    if (rows < 0 || cols <= 0 || dtype < ALCS_F32 || dtype > ALCS_F16) return ALCS_E_INVALID_ARG;
    if (cols > tile::kMaxSize) return ALCS_E_UNSUPPORTED;
    if (rows == 0) return ALCS_OK;
    if (!Y_dev || check_stored(codes_dev, scales_dev) != ALCS_OK) return ALCS_E_INVALID_ARG;
    const int pieces = (cols + 127) / 128 * (dtype == ALCS_F32 ? 32 : 16);
    if (rows > ((1LL << 32) - 512) / pieces) return ALCS_E_UNSUPPORTED;  // a launch has less than 2^32 threads
    const dim3 grid((unsigned)((rows * pieces + 255) / 256));
    const hipStream_t st = (hipStream_t)stream;
    if (dtype == ALCS_F32)
        hipLaunchKernelGGL(k_mx4_dequantize<float>, grid, dim3(256), 0, st, codes_dev, scales_dev, rows, cols, pieces, (float *)Y_dev);
    else if (dtype == ALCS_BF16)
        hipLaunchKernelGGL(k_mx4_dequantize<__bf16>, grid, dim3(256), 0, st, codes_dev, scales_dev, rows, cols, pieces, (__bf16 *)Y_dev);
    else
        hipLaunchKernelGGL(k_mx4_dequantize<_Float16>, grid, dim3(256), 0, st, codes_dev, scales_dev, rows, cols, pieces, (_Float16 *)Y_dev);
    return launched();
}

static int check_linear(int M, int N, int K) {
    if (M < 0 || N <= 0 || K <= 0 || K % 128) return ALCS_E_INVALID_ARG;
    return M > tile::kMaxSize || N > tile::kMaxSize || K / 2 > kNearPitch ? ALCS_E_UNSUPPORTED : ALCS_OK;
}

extern "C" long long alcs_mx4_linear_workspace_bytes(int M, int N, int K) {
    const int rc = check_linear(M, N, K);
    if (rc != ALCS_OK) return rc;
    int cus = 0, xcds = 0;
    if (current_device_shape(&cus, &xcds) != ALCS_OK) return ALCS_E_HIP;
    return few_rows(kMX4, M, N, K, false, cus) ? 0 : plan_tiles(linear_shape(M, N, K), INT64_MAX, cus).workspace;
}

extern "C" int alcs_mx4_linear(const uint8_t *X_codes_dev, const uint8_t *X_scales_dev, const uint8_t *W_codes_dev,
                               const uint8_t *W_scales_dev, const float *bias_dev, void *Y_dev, int M, int N, int K, int dtype,
                               int activation, void *workspace_dev, long long workspace_bytes, void *stream) {
    int rc = check_linear(M, N, K);
    if (rc != ALCS_OK) return rc;
    if (dtype < ALCS_F32 || dtype > ALCS_F16 || activation < ALCS_ACT_NONE || activation > ALCS_ACT_RELU6) return ALCS_E_INVALID_ARG;
    if (M == 0) return ALCS_OK;
    if (!Y_dev || check_stored(X_codes_dev, X_scales_dev) != ALCS_OK || check_stored(W_codes_dev, W_scales_dev) != ALCS_OK)
        return ALCS_E_INVALID_ARG;
    if (workspace_dev && (uintptr_t)workspace_dev % 16) return ALCS_E_INVALID_ARG;
    int cus = 0, xcds = 0;
    if (current_device_shape(&cus, &xcds) != ALCS_OK) return ALCS_E_HIP;
    Args a{};
    a.A[0] = {(const char *)X_codes_dev, K / 2, X_scales_dev, M};
    a.B[0] = {(const char *)W_codes_dev, K / 2, W_scales_dev, N};
    a.M = M; a.N = N; a.KA = a.KB = K;
    a.segs = a.results = 1;
    a.bias[0] = bias_dev;
    a.out[0] = Y_dev;
    a.ldo = N;
    a.act = activation;
    const hipStream_t st = (hipStream_t)stream;
    if (dtype == ALCS_F32) return linear_as<float>(a, workspace_dev, workspace_bytes, cus, xcds, st);
    if (dtype == ALCS_BF16) return linear_as<__bf16>(a, workspace_dev, workspace_bytes, cus, xcds, st);
    return linear_as<_Float16>(a, workspace_dev, workspace_bytes, cus, xcds, st);
}
