// The gated feed-forward block and its gradients (alcs.h): the two projections, the gate and the product in one
// kernel, alcs_tile.h's; the backward pass is one pass over [T, F] and two launches of the same kernel.
#include "alcs_tile.h"

namespace alcs {
namespace tile {

// ------------------------------------------------------------------------------ gradients at the gate

// dU = dH * gate(G), dG = dH * U * gate'(G) for a strip of columns and a part of the rows, four neighbouring
// columns a thread, and the sums of both over those rows (for the biases' gradients, from the values before
// they are rounded).  Bound by memory: three tensors in, two out.  The results' rows are padded with zeros to
// whole 16-byte pieces, which the products behind read.
struct GradArgs {
    const void *G, *U, *dH;
    void *dG, *dU;
    float *sums;         // [part][2][F] or null
    int T, F, pitch;     // pitch of dG and dU, elements
    int rows, gate, vec; // rows of a part; vec: G, U, dH may be read four elements at a time
};

template <class T> __device__ inline void load4(const T *p, int n, int vec, float v[4]) {
    if (vec && n >= 4) {
        struct alignas(sizeof(T) * 4) Four { T e[4]; };
        const Four f = *(const Four *)p;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = to_float(f.e[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = i < n ? to_float(p[i]) : 0.0f;
    }
}

template <class T> __global__ __launch_bounds__(256) void k_gate_grad(const GradArgs a) {
    __shared__ float join[4][64][8];
    const int x = threadIdx.x & 63, y = threadIdx.x >> 6;
    const int c = (blockIdx.x * 64 + x) * 4;
    const int r0 = blockIdx.y * a.rows, r1 = min(r0 + a.rows, a.T);
    float sg[4] = {}, su[4] = {};
    if (c < a.pitch) {
        const int n = a.F - c;
#pragma clang loop unroll_count(4)
        for (int r = r0 + y; r < r1; r += 4) {
            const long long at = (long long)r * a.F + c;
            float g[4], u[4], h[4], dg[4], du[4];
            load4((const T *)a.G + at, n, a.vec, g);
            load4((const T *)a.U + at, n, a.vec, u);
            load4((const T *)a.dH + at, n, a.vec, h);
            float v[4], d[4];
            gate_slopes<sizeof(T) == 4>(a.gate, g, v, d);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                du[i] = i < n ? h[i] * v[i] : 0.0f;
                dg[i] = i < n ? h[i] * u[i] * d[i] : 0.0f;
                sg[i] += dg[i];
                su[i] += du[i];
            }
            store4((T *)a.dG + (long long)r * a.pitch + c, dg, 4, 1);
            store4((T *)a.dU + (long long)r * a.pitch + c, du, 4, 1);
        }
    }
    if (!a.sums) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) { join[y][x][i] = sg[i]; join[y][x][4 + i] = su[i]; }
    __syncthreads();
    // 64 * 4 columns of two planes, two values a thread
    for (int j = threadIdx.x; j < 512; j += 256) {
        const int plane = j >> 8, col = j & 255, n = blockIdx.x * 256 + col;
        if (n >= a.F) continue;
        float s = 0.0f;
#pragma unroll
        for (int k = 0; k < 4; ++k) s += join[k][col >> 2][plane * 4 + (col & 3)];
        a.sums[((long long)blockIdx.y * 2 + plane) * a.F + n] = s;
    }
}
// The parts' sums: 32 columns and eight shares of the parts a workgroup, each added in the order of the parts, the
// shares in theirs.
template <class T> __global__ __launch_bounds__(256) void k_bias_grad(const float *sums, int parts, int F, T *dbg, T *dbu) {
    __shared__ float join[8][32];
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    const long long at = (long long)blockIdx.x * 32 + x;
    float s = 0.0f;
    if (at < 2LL * F) {
        const int from = (int)((long long)parts * y / 8), to = (int)((long long)parts * (y + 1) / 8);
#pragma clang loop unroll_count(8)
        for (int k = from; k < to; ++k) s += sums[(long long)k * 2 * F + at];
    }
    join[y][x] = s;
    __syncthreads();
    if (y || at >= 2LL * F) return;
#pragma unroll
    for (int k = 1; k < 8; ++k) s += join[k][x];
    T *out = at < F ? dbg : dbu;
    if (out) out[at % F] = (T)s;
}
template <class T> __global__ __launch_bounds__(256) void k_fill_zero(T *p, long long n) {
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) p[i] = (T)0.0f;
}
template <class T> int fill_zero(void *p, long long n, hipStream_t stream) {
    if (!p) return ALCS_OK;
    const long long blocks = std::min<long long>((n + 255) / 256, 1 << 16);
    hipLaunchKernelGGL((k_fill_zero<T>), dim3((unsigned)blocks), dim3(256), 0, stream, (T *)p, n);
    return launched();
}

// ------------------------------------------------------------------------------ host side

constexpr int kMaxSize = 1 << 28;  // rows, columns: tile and piece numbers stay far inside 31 bits

// Rows that the direct loads take: they start at 16-byte addresses and hold whole 16-byte pieces.
inline bool aligned_rows(const void *p, long long ld, int columns, int E, int rows) {
    const int n = per16(E);
    return (uintptr_t)p % 16 == 0 && columns % n == 0 && (ld % n == 0 || rows <= 1);
}

inline Shape forward_shape(int E, int T, int D, int F) { return {E, true, false, false, T, F, D, 1, 1}; }
inline Shape dx_shape(int E, int T, int D, int pitch) { return {E, false, false, true, T, D, pitch, 2, 1}; }
inline Shape dw_shape(int E, int T, int D, int F) { return {E, false, true, true, F, D, T, 1, 2}; }

template <int E> int gated_as(Args a, bool aligned, void *workspace, long long workspace_bytes, int cus, int xcds, hipStream_t stream) {
    typedef typename TypeOf<E>::type T;
    if (few_rows(a.M, a.N, cus)) return launch_few<E, T, true>(a, aligned, stream);
    const bool near = aligned && near_rows({a.A[0].pitch, a.B[0].pitch, a.B[1].pitch});
    const Plan p = plan_tiles(forward_shape(E, a.M, a.KA, a.N), near, workspace ? workspace_bytes : 0, cus);
    return launch_tiles<E, T, false, false, true>(a, p, aligned, workspace, cus, xcds, stream);
}

struct BackwardSpace {  // bytes from the start of the workspace
    int pitch;          // of dG and dU, elements
    long long dG, dU, sums, partial, total;
    int parts, rows;
};
inline BackwardSpace backward_space(int T, int D, int F, int E, int cus) {
    BackwardSpace s{};
    const int n = per16(E);
    s.pitch = (F + n - 1) / n * n;
    const long long each = ((long long)T * s.pitch * bytes_of(E) + 255) / 256 * 256;
    // parts of 64 rows, longer ones where there are more than 1024; of 16 (all of a thread's loads in flight at once)
    // where that makes no more workgroups than the card runs together: 333 x 2730, bfloat16, 5 us, not 23
    const long long strips = (s.pitch + 255) / 256;
    s.rows = strips * ((T + 15) / 16) <= 8LL * cus ? 16 : std::max(64, (T + 1023) / 1024);
    s.parts = (T + s.rows - 1) / s.rows;
    s.dG = 0;
    s.dU = each;
    s.sums = 2 * each;
    s.partial = s.sums + ((long long)s.parts * 2 * F * 4 + 255) / 256 * 256;
    s.total = s.partial + std::max(workspace_of(dx_shape(E, T, D, s.pitch), cus), workspace_of(dw_shape(E, T, D, F), cus));
    return s;
}

struct BackwardArgs {
    const void *X, *Wg, *Wu, *G, *U, *dH;
    long long ldx, ldg, ldu;
    void *dX, *dWg, *dWu, *dbg, *dbu;
    int T, D, F, gate;
};
template <int E> int backward_as(const BackwardArgs &b, char *workspace, int cus, int xcds, hipStream_t stream) {
    typedef typename TypeOf<E>::type T;
    int rc;
    if (b.T == 0) {  // sums over no rows
        if ((rc = fill_zero<T>(b.dWg, (long long)b.F * b.D, stream)) != ALCS_OK) return rc;
        if ((rc = fill_zero<T>(b.dWu, (long long)b.F * b.D, stream)) != ALCS_OK) return rc;
        if ((rc = fill_zero<T>(b.dbg, b.F, stream)) != ALCS_OK) return rc;
        return fill_zero<T>(b.dbu, b.F, stream);
    }
    const BackwardSpace s = backward_space(b.T, b.D, b.F, E, cus);
    GradArgs g{};
    g.G = b.G; g.U = b.U; g.dH = b.dH;
    g.dG = workspace + s.dG; g.dU = workspace + s.dU;
    g.sums = b.dbg || b.dbu ? (float *)(workspace + s.sums) : nullptr;
    g.T = b.T; g.F = b.F; g.pitch = s.pitch; g.rows = s.rows; g.gate = b.gate;
    const uintptr_t where = (uintptr_t)b.G | (uintptr_t)b.U | (uintptr_t)b.dH;
    g.vec = b.F % 4 == 0 && where % (4 * sizeof(T)) == 0;
    hipLaunchKernelGGL((k_gate_grad<T>), dim3((unsigned)((s.pitch + 255) / 256), (unsigned)s.parts), dim3(256), 0, stream, g);
    if ((rc = launched()) != ALCS_OK) return rc;
    if (g.sums) {
        hipLaunchKernelGGL((k_bias_grad<T>), dim3((unsigned)((2LL * b.F + 31) / 32)), dim3(256), 0, stream, g.sums, s.parts, b.F,
                           (T *)b.dbg, (T *)b.dbu);
        if ((rc = launched()) != ALCS_OK) return rc;
    }
    const long long sz = bytes_of(E), pitch = s.pitch * sz;
    if (b.dX) {  // dX = dG Wg + dU Wu: one sum over two segments
        Args a{};
        a.A[0] = {(const char *)g.dG, pitch, nullptr, b.T};
        a.A[1] = {(const char *)g.dU, pitch, nullptr, b.T};
        a.B[0] = {(const char *)b.Wg, b.ldg * sz, nullptr, b.D};
        a.B[1] = {(const char *)b.Wu, b.ldu * sz, nullptr, b.D};
        a.M = b.T; a.N = b.D; a.KA = s.pitch; a.KB = b.F;
        a.segs = 2; a.results = 1;
        a.out[0] = b.dX;
        a.ldo = b.D;
        a.vec = rows_of_eights({b.dX}, b.D);
        const bool al = aligned_rows(b.Wg, b.ldg, b.D, E, b.F) && aligned_rows(b.Wu, b.ldu, b.D, E, b.F);
        const Plan p = plan_tiles(dx_shape(E, b.T, b.D, s.pitch), al && near_rows({pitch, b.ldg * sz, b.ldu * sz}), INT64_MAX, cus);
        if ((rc = launch_tiles<E, T, false, true, false>(a, p, al, workspace + s.partial, cus, xcds, stream)) != ALCS_OK) return rc;
    }
    if (b.dWg) {  // dWg = dG^T X and dWu = dU^T X
        Args a{};
        a.A[0] = {(const char *)g.dG, pitch, nullptr, s.pitch};
        a.A[1] = {(const char *)g.dU, pitch, nullptr, s.pitch};
        a.B[0] = a.B[1] = {(const char *)b.X, b.ldx * sz, nullptr, b.D};
        a.M = b.F; a.N = b.D; a.KA = a.KB = b.T;
        a.segs = 1; a.results = 2;
        a.out[0] = b.dWg; a.out[1] = b.dWu;
        a.ldo = b.D;
        a.vec = rows_of_eights({b.dWg, b.dWu}, b.D);
        const bool al = aligned_rows(b.X, b.ldx, b.D, E, b.T);
        const Plan p = plan_tiles(dw_shape(E, b.T, b.D, b.F), al && near_rows({pitch, b.ldx * sz}), INT64_MAX, cus);
        if ((rc = launch_tiles<E, T, true, true, false>(a, p, al, workspace + s.partial, cus, xcds, stream)) != ALCS_OK) return rc;
    }
    return ALCS_OK;
}

int check(int T, int D, int F, int dtype, int gate) {
    if (T < 0 || D <= 0 || F <= 0) return ALCS_E_INVALID_ARG;
    if (dtype < ALCS_F32 || dtype > ALCS_F16 || gate < ALCS_GATE_NONE || gate > ALCS_GATE_SIGMOID) return ALCS_E_INVALID_ARG;
    return T > kMaxSize || D > kMaxSize || F > kMaxSize ? ALCS_E_UNSUPPORTED : ALCS_OK;
}

}  // namespace tile
}  // namespace alcs

using namespace alcs;
using namespace alcs::tile;

extern "C" long long alcs_gated_ff_workspace_bytes(int T, int D, int F, int dtype) {
    int cus = 0, xcds = 0;
    const int rc = check(T, D, F, dtype, 0);
    if (rc != ALCS_OK) return rc;
    if (current_device_shape(&cus, &xcds) != ALCS_OK) return ALCS_E_HIP;
    return few_rows(T, F, cus) ? 0 : workspace_of(forward_shape(dtype, T, D, F), cus);
}
extern "C" long long alcs_gated_ff_backward_workspace_bytes(int T, int D, int F, int dtype) {
    int cus = 0, xcds = 0;
    const int rc = check(T, D, F, dtype, 0);
    if (rc != ALCS_OK) return rc;
    if (current_device_shape(&cus, &xcds) != ALCS_OK) return ALCS_E_HIP;
    return T == 0 ? 0 : backward_space(T, D, F, dtype, cus).total;
}

extern "C" int alcs_gated_ff(const void *X_dev, long long ldx, const void *Wg_dev, long long ldg, const void *Wu_dev, long long ldu,
                             const float *bg_dev, const float *bu_dev, void *H_dev, void *G_dev, void *U_dev, int T, int D, int F,
                             int dtype, int gate, void *workspace_dev, long long workspace_bytes, void *stream) {
    int rc = check(T, D, F, dtype, gate);
    if (rc != ALCS_OK) return rc;
    if (ldx < 0 || ldg < 0 || ldu < 0 || !G_dev != !U_dev || (uintptr_t)workspace_dev % 16) return ALCS_E_INVALID_ARG;
    if (T == 0) return ALCS_OK;
    if (!X_dev || !Wg_dev || !Wu_dev || !H_dev) return ALCS_E_INVALID_ARG;
    int cus = 0, xcds = 0;
    if (current_device_shape(&cus, &xcds) != ALCS_OK) return ALCS_E_HIP;
    const long long sz = dtype == ALCS_F32 ? 4 : 2;
    Args a{};
    a.A[0] = {(const char *)X_dev, ldx * sz, nullptr, T};
    a.B[0] = {(const char *)Wg_dev, ldg * sz, nullptr, F};
    a.B[1] = {(const char *)Wu_dev, ldu * sz, nullptr, F};
    a.M = T; a.N = F; a.KA = a.KB = D;
    a.segs = a.results = 1;
    a.bias[0] = bg_dev; a.bias[1] = bu_dev;
    a.out[0] = H_dev; a.pre[0] = G_dev; a.pre[1] = U_dev;
    a.ldo = F;
    a.act = gate;
    a.vec = rows_of_eights({H_dev, G_dev, U_dev}, F);
    const bool al = aligned_rows(X_dev, ldx, D, dtype, T) && aligned_rows(Wg_dev, ldg, D, dtype, F) &&
                    aligned_rows(Wu_dev, ldu, D, dtype, F);
    const hipStream_t st = (hipStream_t)stream;
    if (dtype == ALCS_F32) return gated_as<kF32>(a, al, workspace_dev, workspace_bytes, cus, xcds, st);
    if (dtype == ALCS_BF16) return gated_as<kBF16>(a, al, workspace_dev, workspace_bytes, cus, xcds, st);
    return gated_as<kF16>(a, al, workspace_dev, workspace_bytes, cus, xcds, st);
}

extern "C" int alcs_gated_ff_backward(const void *X_dev, long long ldx, const void *Wg_dev, long long ldg, const void *Wu_dev,
                                      long long ldu, const void *G_dev, const void *U_dev, const void *dH_dev, void *dX_dev,
                                      void *dWg_dev, void *dWu_dev, void *dbg_dev, void *dbu_dev, int T, int D, int F, int dtype,
                                      int gate, void *workspace_dev, long long workspace_bytes, void *stream) {
    int rc = check(T, D, F, dtype, gate);
    if (rc != ALCS_OK) return rc;
    if (ldx < 0 || ldg < 0 || ldu < 0 || !dWg_dev != !dWu_dev || !dbg_dev != !dbu_dev) return ALCS_E_INVALID_ARG;
    if (T > 0 && (!X_dev || !Wg_dev || !Wu_dev || !G_dev || !U_dev || !dH_dev)) return ALCS_E_INVALID_ARG;
    int cus = 0, xcds = 0;
    if (current_device_shape(&cus, &xcds) != ALCS_OK) return ALCS_E_HIP;
    if (T > 0 && (!workspace_dev || (uintptr_t)workspace_dev % 16 || workspace_bytes < backward_space(T, D, F, dtype, cus).total))
        return ALCS_E_INVALID_ARG;
    const BackwardArgs b = {X_dev, Wg_dev, Wu_dev, G_dev, U_dev, dH_dev, ldx, ldg, ldu, dX_dev, dWg_dev, dWu_dev, dbg_dev, dbu_dev,
                            T, D, F, gate};
    const hipStream_t st = (hipStream_t)stream;
    if (dtype == ALCS_F32) return backward_as<kF32>(b, (char *)workspace_dev, cus, xcds, st);
    if (dtype == ALCS_BF16) return backward_as<kBF16>(b, (char *)workspace_dev, cus, xcds, st);
    return backward_as<kF16>(b, (char *)workspace_dev, cus, xcds, st);
}
