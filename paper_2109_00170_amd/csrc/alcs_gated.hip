// The gated feed-forward block and its gradients (alcs.h): the two projections, the gate and the product in one
// kernel, alcs_tile.h's, before it a copy of rows that are not aligned, behind it the sums of a K that was shared out; the
// backward pass is one pass over [T, F] and the products behind it, in one launch or two, with the same around them.
#include "alcs_tile.h"

namespace alcs {
namespace tile {

// ------------------------------------------------------------------------------ gradients at the gate

// dU = dH * gate(G), dG = dH * U * gate'(G) for a strip of columns and a part of the rows, four neighbouring
// columns a thread, and the sums of both over those rows (for the biases' gradients, from the values before
// they are rounded).  Bound by memory: three tensors in, two out.  The results' rows are padded with zeros to
// whole 16-byte pieces, which the products behind read.
// Of 16-bit tensors G and U come, and dG and dU go, in 16 bits: half the bytes of this pass and of what a program keeps
// between forward and backward, and operands that the 16-bit matrix instructions take as they are (two halves of each would
// double the products' work).  Each rounding is half a step of the type at most; together they take the gradients of
// 8192 x 4096, 8192 (bfloat16) from 0.0017 of their norm, the rounding of the results alone, to 0.0031.
struct GradArgs {
    const void *G, *U, *dH;
    void *dG, *dU;
    float *sums;         // [part][2][F] or null
    int T, F, pitch;     // pitch of dG and dU, elements
    int rows, gate;      // rows of a part
};

template <class T> __device__ inline void load4(const T *p, int n, float v[4]) {
    if (n >= 4) {  // of any alignment
        T e[4];
        __builtin_memcpy(e, p, sizeof(e));
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = to_float(e[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = i < n ? to_float(p[i]) : 0.0f;
    }
}

// AHEAD: a thread's rows whose loads are in flight together.
template <class T, int AHEAD> __global__ __launch_bounds__(256) void k_gate_grad(const GradArgs a) {
    __shared__ float join[4][64][9];  // (8 of them; 9 for the banks)
    const int x = threadIdx.x & 63, y = threadIdx.x >> 6;
    const int c = (blockIdx.x * 64 + x) * 4;
    const int r0 = blockIdx.y * a.rows, r1 = min(r0 + a.rows, a.T);
    float sg[4] = {}, su[4] = {};
    if (c < a.pitch) {
        const int n = a.F - c;
#pragma clang loop unroll_count(AHEAD)
        for (int r = r0 + y; r < r1; r += 4) {
            const long long at = (long long)r * a.F + c;
            float g[4], u[4], h[4], dg[4], du[4];
            load4((const T *)a.G + at, n, g);
            load4((const T *)a.U + at, n, u);
            load4((const T *)a.dH + at, n, h);
            float v[4], d[4];
            gate_slopes<sizeof(T) == 4>(a.gate, g, v, d);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                du[i] = i < n ? h[i] * v[i] : 0.0f;
                dg[i] = i < n ? h[i] * (u[i] * d[i]) : 0.0f;  // (u * d first: with a slope of 0 no product overflows)
                sg[i] += dg[i];
                su[i] += du[i];
            }
            store_some<4>((T *)a.dG + (long long)r * a.pitch + c, dg, 4);
            store_some<4>((T *)a.dU + (long long)r * a.pitch + c, du, 4);
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
template <class T> __global__ __launch_bounds__(256) void k_bias_grad(const BiasArgs a) {
    __shared__ float lds[256];
    bias_tile<T>(a, blockIdx.x, lds);
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

constexpr int kMaxRows = 1 << 26;  // numbers of rows and threads stay inside 32 bits
constexpr int kMaxWidth = 1 << 20;  // D and F: rows of copies, of dG and of dU are near ones, in float32 too
static_assert(kMaxWidth * 4LL <= kNearPitch, "a tile's offsets are 32 bits");

// Rows that the tiles' direct loads take: they start at 16-byte addresses, hold whole 16-byte pieces and lie at most
// kNearPitch apart.
inline bool near_rows(const void *p, long long ld, int columns, int E, int rows) {
    const int n = per16(E);
    return (uintptr_t)p % 16 == 0 && columns % n == 0 && (rows <= 1 || (ld % n == 0 && ld * bytes_of(E) <= kNearPitch));
}

// Copies of up to three matrices whose rows the tiles do not take, padded with zeros to whole pieces: a wavefront a row.
// 2000 x 999 -> 2 x 2731 (bfloat16) 41 + 9 us, where tiles that read odd rows themselves, through registers,
// took 69.
struct AlignArgs {
    const char *from[3];
    long long pitch[3];  // bytes
    char *to[3];
    int rows[3];
    int columns, pieces;
};
template <class T> __global__ __launch_bounds__(256) void k_align(const AlignArgs a) {
    constexpr int n = 16 / sizeof(T);
    const int all = a.rows[0] + a.rows[1] + a.rows[2];
    for (int at = (int)blockIdx.x * 4 + (int)(threadIdx.x >> 6); at < all; at += (int)gridDim.x * 4) {
        int row = at, i = 0;
        if (row >= a.rows[0]) { row -= a.rows[0]; i = 1; }
        if (i == 1 && row >= a.rows[1]) { row -= a.rows[1]; i = 2; }
        const char *from = (i == 0 ? a.from[0] : i == 1 ? a.from[1] : a.from[2]) + row * (i == 0 ? a.pitch[0] : i == 1 ? a.pitch[1] : a.pitch[2]);
        char *to = (i == 0 ? a.to[0] : i == 1 ? a.to[1] : a.to[2]) + (long long)row * a.pieces * 16;
        for (int c = threadIdx.x & 63; c < a.pieces; c += 64) {
            v4i v = {0, 0, 0, 0};
            const int left = a.columns - c * n;
            if (left >= n) {
                __builtin_memcpy(&v, from + (long long)c * 16, 16);
            } else {
                T e[n] = {};
#pragma unroll
                for (int j = 0; j < n; ++j)
                    if (j < left) __builtin_memcpy(&e[j], from + (long long)c * 16 + j * sizeof(T), sizeof(T));
                __builtin_memcpy(&v, e, 16);
            }
            *(v4i *)(to + (long long)c * 16) = v;
        }
    }
}
// Those of the operands that are not near go to `space` (room for all of them); their pointers and pitches follow.
template <int E> int align_rows(std::initializer_list<Operand *> operands, std::initializer_list<int> rows, int columns, char *space, hipStream_t stream) {
    typedef typename TypeOf<E>::type T;
    AlignArgs g{};
    g.columns = columns;
    g.pieces = whole_pieces(columns, E) / per16(E);
    int n = 0;
    long long total = 0;
    const int *r = rows.begin();
    for (Operand *o : operands) {
        const int count = *r++;
        if (near_rows(o->p, o->pitch / bytes_of(E), columns, E, count)) continue;
        g.from[n] = o->p;
        g.pitch[n] = o->pitch;
        g.to[n] = space;
        g.rows[n++] = count;
        o->p = space;
        o->pitch = g.pieces * 16LL;
        space += whole256((long long)count * g.pieces * 16);
        total += count;
    }
    if (!n) return ALCS_OK;
    hipLaunchKernelGGL((k_align<T>), dim3((unsigned)std::min((total + 3) / 4, 1LL << 16)), dim3(256), 0, stream, g);
    return launched();
}

inline long long copy_bytes(int rows, int D, int E) { return whole256((long long)rows * whole_pieces(D, E) * bytes_of(E)); }
inline long long forward_copies(int E, int T, int D, int F) { return copy_bytes(T, D, E) + 2 * copy_bytes(F, D, E); }

template <int E> int gated_as(Args a, char *workspace, long long workspace_bytes, int cus, int xcds, hipStream_t stream) {
    typedef typename TypeOf<E>::type T;
    const int D = a.KA;
    const int n = per16(E);
    const bool aligned = D % n == 0 && (uintptr_t)a.A[0].p % 16 == 0 && (uintptr_t)a.B[0].p % 16 == 0 && (uintptr_t)a.B[1].p % 16 == 0 &&
                         a.A[0].pitch % 16 == 0 && a.B[0].pitch % 16 == 0 && a.B[1].pitch % 16 == 0;
    if (few_rows(E, a.M, a.N, D, true, cus)) return launch_few<E, T, true>(a, aligned, stream);
    const long long sz = bytes_of(E);
    const bool near = near_rows(a.A[0].p, a.A[0].pitch / sz, D, E, a.M) && near_rows(a.B[0].p, a.B[0].pitch / sz, D, E, a.N) &&
                      near_rows(a.B[1].p, a.B[1].pitch / sz, D, E, a.N);
    if (!workspace) workspace_bytes = 0;
    if (!near) {
        const long long copies = forward_copies(E, a.M, D, a.N);
        if (workspace_bytes < copies) return launch_few<E, T, true>(a, aligned, stream);
        const int rc = align_rows<E>({&a.A[0], &a.B[0], &a.B[1]}, {a.M, a.N, a.N}, D, workspace, stream);
        if (rc != ALCS_OK) return rc;
        workspace += copies;
        workspace_bytes -= copies;
        a.KA = a.KB = whole_pieces(D, E);
    }
    const Plan p = plan_tiles(forward_shape(E, a.M, a.KA, a.N), workspace_bytes, cus);
    return launch_tiles<E, T, false, false, true>(a, p, workspace, cus, xcds, stream);
}

struct BackwardSpace {  // bytes from the start of the workspace
    int pitch;          // of dG and dU, elements
    long long dG, dU, sums, copies, partial, total;
    int parts, rows;
    Plans plans;
};
inline BackwardSpace backward_space(int T, int D, int F, int E, int cus) {
    BackwardSpace s{};
    s.pitch = whole_pieces(F, E);
    const long long each = whole256((long long)T * s.pitch * bytes_of(E));
    // parts of 64 rows, longer ones where there are more than 1024; of 16 (all of a thread's loads in flight at once)
    // where that makes no more workgroups than the card runs together: 333 x 2730, bfloat16, 7 us, not 23
    const long long strips = (s.pitch + 255) / 256;
    s.rows = strips * ((T + 15) / 16) <= 8LL * cus ? 16 : std::max(64, (T + 1023) / 1024);
    s.parts = (T + s.rows - 1) / s.rows;
    s.dG = 0;
    s.dU = each;
    s.sums = 2 * each;
    s.copies = s.sums + whole256((long long)s.parts * 2 * F * 4);
    s.partial = s.copies + forward_copies(E, T, D, F);
    s.plans = plan_pair(dx_shape(E, T, D, s.pitch), dw_shape(E, T, D, F), cus);
    s.total = s.partial + s.plans.workspace;
    return s;
}

struct BackwardArgs {
    const void *X, *Wg, *Wu, *G, *U, *dH;
    long long ldx, ldg, ldu;
    void *dX, *dWg, *dWu, *dbg, *dbu;
    int T, D, F, gate;
};
template <int E> int backward_as(const BackwardArgs &b, char *workspace, long long workspace_bytes, int cus, int xcds, hipStream_t stream) {
    typedef typename TypeOf<E>::type T;
    int rc;
    if (b.T == 0) {  // sums over no rows
        if ((rc = fill_zero<T>(b.dWg, (long long)b.F * b.D, stream)) != ALCS_OK) return rc;
        if ((rc = fill_zero<T>(b.dWu, (long long)b.F * b.D, stream)) != ALCS_OK) return rc;
        if ((rc = fill_zero<T>(b.dbg, b.F, stream)) != ALCS_OK) return rc;
        return fill_zero<T>(b.dbu, b.F, stream);
    }
    const BackwardSpace s = backward_space(b.T, b.D, b.F, E, cus);
    if (!workspace || (uintptr_t)workspace % 16 || workspace_bytes < s.total) return ALCS_E_INVALID_ARG;
    GradArgs g{};
    g.G = b.G; g.U = b.U; g.dH = b.dH;
    g.dG = workspace + s.dG; g.dU = workspace + s.dU;
    g.sums = b.dbg || b.dbu ? (float *)(workspace + s.sums) : nullptr;
    g.T = b.T; g.F = b.F; g.pitch = s.pitch; g.rows = s.rows; g.gate = b.gate;
    // (many parts have wavefronts enough: 8192 x 8192, bfloat16, 123 us with one row ahead, 154 with four)
    auto grad = s.rows == 16 ? k_gate_grad<T, 4> : k_gate_grad<T, 1>;
    hipLaunchKernelGGL(grad, dim3((unsigned)((s.pitch + 255) / 256), (unsigned)s.parts), dim3(256), 0, stream, g);
    if ((rc = launched()) != ALCS_OK) return rc;
    BiasArgs bias{g.sums, s.parts, b.F, b.dbg, b.dbu, g.sums ? (unsigned)((2LL * b.F + 31) / 32) : 0};
    const bool together = s.plans.together && b.dX && b.dWg;
    if (g.sums && !together) {
        hipLaunchKernelGGL((k_bias_grad<T>), dim3(bias.blocks), dim3(256), 0, stream, bias);
        if ((rc = launched()) != ALCS_OK) return rc;
    }
    const long long sz = bytes_of(E), pitch = s.pitch * sz;
    const int columns = whole_pieces(b.D, E);
    Args x{}, w{};
    if (b.dX) {  // dX = dG Wg + dU Wu: one sum over two segments
        x.A[0] = {(const char *)g.dG, pitch, nullptr, b.T};
        x.A[1] = {(const char *)g.dU, pitch, nullptr, b.T};
        x.B[0] = {(const char *)b.Wg, b.ldg * sz, nullptr, columns};
        x.B[1] = {(const char *)b.Wu, b.ldu * sz, nullptr, columns};
        x.M = b.T; x.N = b.D; x.KA = s.pitch; x.KB = b.F;
        x.segs = 2; x.results = 1;
        x.out[0] = b.dX;
        x.ldo = b.D;
    }
    if (b.dWg) {  // dWg = dG^T X and dWu = dU^T X
        w.A[0] = {(const char *)g.dG, pitch, nullptr, s.pitch};
        w.A[1] = {(const char *)g.dU, pitch, nullptr, s.pitch};
        w.B[0] = {(const char *)b.X, b.ldx * sz, nullptr, columns};
        w.M = b.F; w.N = b.D; w.KA = w.KB = b.T;
        w.segs = 1; w.results = 2;
        w.out[0] = b.dWg; w.out[1] = b.dWu;
        w.ldo = b.D;
    }
    char *copies = workspace + s.copies, *partial = workspace + s.partial;
    if (b.dX && b.dWg) rc = align_rows<E>({&x.B[0], &x.B[1], &w.B[0]}, {b.F, b.F, b.T}, b.D, copies, stream);
    else if (b.dX) rc = align_rows<E>({&x.B[0], &x.B[1]}, {b.F, b.F}, b.D, copies, stream);
    else if (b.dWg) rc = align_rows<E>({&w.B[0]}, {b.T}, b.D, copies, stream);
    if (rc != ALCS_OK) return rc;
    w.B[1] = w.B[0];
    const Shape sx = dx_shape(E, b.T, b.D, s.pitch), sw = dw_shape(E, b.T, b.D, b.F);
    if (together) return launch_pair<E, T>(x, w, bias, sx, sw, s.plans, partial, xcds, stream);
    if (b.dX && (rc = launch_tiles<E, T, false, true, false>(x, plan_tiles(sx, s.plans.workspace, cus), partial, cus, xcds, stream)) != ALCS_OK) return rc;
    return b.dWg ? launch_tiles<E, T, true, true, false>(w, plan_tiles(sw, s.plans.workspace, cus), partial, cus, xcds, stream) : ALCS_OK;
}

int check(int T, int D, int F, int dtype, int gate) {
    if (T < 0 || D <= 0 || F <= 0) return ALCS_E_INVALID_ARG;
    if (dtype < ALCS_F32 || dtype > ALCS_F16 || gate < ALCS_GATE_NONE || gate > ALCS_GATE_SIGMOID) return ALCS_E_INVALID_ARG;
    return T > kMaxRows || D > kMaxWidth || F > kMaxWidth ? ALCS_E_UNSUPPORTED : ALCS_OK;
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
    if (few_rows(dtype, T, F, D, true, cus)) return 0;
    return (D % per16(dtype) ? forward_copies(dtype, T, D, F) : 0) + plan_tiles(forward_shape(dtype, T, whole_pieces(D, dtype), F), INT64_MAX, cus).workspace;
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
    const hipStream_t st = (hipStream_t)stream;
    if (dtype == ALCS_F32) return gated_as<kF32>(a, (char *)workspace_dev, workspace_bytes, cus, xcds, st);
    if (dtype == ALCS_BF16) return gated_as<kBF16>(a, (char *)workspace_dev, workspace_bytes, cus, xcds, st);
    return gated_as<kF16>(a, (char *)workspace_dev, workspace_bytes, cus, xcds, st);
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
    const BackwardArgs b = {X_dev, Wg_dev, Wu_dev, G_dev, U_dev, dH_dev, ldx, ldg, ldu, dX_dev, dWg_dev, dWu_dev, dbg_dev, dbu_dev,
                            T, D, F, gate};
    const hipStream_t st = (hipStream_t)stream;
    if (dtype == ALCS_F32) return backward_as<kF32>(b, (char *)workspace_dev, workspace_bytes, cus, xcds, st);
    if (dtype == ALCS_BF16) return backward_as<kBF16>(b, (char *)workspace_dev, workspace_bytes, cus, xcds, st);
    return backward_as<kF16>(b, (char *)workspace_dev, workspace_bytes, cus, xcds, st);
}
