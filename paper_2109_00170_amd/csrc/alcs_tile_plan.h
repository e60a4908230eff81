// Which kernels of alcs_tile.h a product of the feed-forward layers runs: host arithmetic alone, so that a test can ask
// for it without a GPU.
#pragma once
#include <algorithm>
#include <cstdint>

#include "alcs.h"

namespace alcs {
namespace tile {

enum Elem { kF32 = ALCS_F32, kBF16 = 1, kF16 = 2, kMX4 = 3 };
constexpr int bytes_of(int E) { return E == kF32 ? 4 : 2; }                  // not for kMX4
constexpr int per16(int E) { return E == kF32 ? 4 : E == kMX4 ? 32 : 8; }    // elements in 16 bytes
constexpr int kTileBytes = 128;                                              // of K, per row

// Rows of sums start at 16-byte addresses.
constexpr int sum_pitch(int n) { return (n + 3) & ~3; }

// Kinds of tiles: 256 x 256 (k_big), 128 x 128 and 64 x 128 (k_mid).
enum Kind { kBig = 0, k128 = 1, k64 = 2 };
struct Plan {
    int kind, tiles_m, tiles_n, ktiles, splits;
    long long workspace;  // bytes of sums that a split needs
};
struct Shape {
    int E;
    bool gated, strided;  // strided: the sum runs over the rows of B, or of both
    long long M, N, K;  // rows, columns (of each projection where gated), elements of K in a segment
    int segs, results;
};
inline long long up(long long a, long long b) { return (a + b - 1) / b; }
inline int whole_pieces(int columns, int E) { return (columns + per16(E) - 1) / per16(E) * per16(E); }
inline Shape linear_shape(int M, int N, int K) { return {kMX4, false, false, M, N, K, 1, 1}; }
inline Shape forward_shape(int E, int T, int D, int F) { return {E, true, false, T, F, D, 1, 1}; }
inline Shape dx_shape(int E, int T, int D, int pitch) { return {E, false, true, T, D, pitch, 2, 1}; }
inline Shape dw_shape(int E, int T, int D, int F) { return {E, false, true, F, D, T, 1, 2}; }
inline Plan plan_of(const Shape &s, int kind, int splits) {
    Plan p{};
    p.kind = kind;
    const int rows = kind == kBig ? 256 : kind == k64 ? 64 : 128, cols = kind == kBig ? 256 : 128;
    p.ktiles = (int)up(s.K, 8 * per16(s.E));
    p.tiles_m = (int)up(s.M, rows);
    p.tiles_n = (int)up(s.N, s.gated ? cols / 2 : cols);
    p.splits = splits;
    p.workspace = splits > 1 ? (long long)splits * (s.gated ? 2 : s.results) * s.M * sum_pitch((int)s.N) * 4 : 0;
    return p;
}
// What a plan takes, in microseconds, as measured on MI355X: a launch with its first loads and its stores, then so much
// for a K tile of 128 bytes a row, of one workgroup alone on its compute unit and of two.  Small tiles of 16 bits
// alone: 0.32 and 0.50; where the sum runs over rows (transposing reads) a third more; 256 x 256 tiles run at the
// card's power limit.  A split costs another launch and the sums' way out and back at 8 TB/s (they
// stay in the last cache, where the operands were too for the first three lines: as a layer finds them behind others).
//   333 x 1000 -> 2 x 2730 (bfloat16): 64 rows (258 tiles) 14.5 us, 128 x 128 16.9; from memory 16.9 and 21.8, from L2 15.0 and 13.2
//   500 x 2000 -> 2 x 2200 (bfloat16): 64 rows (280 tiles) 26.5 us, 128 x 128 23.1
//   700 x 1024 -> 2 x 4096 (bfloat16): 64 rows (704 tiles) 20.3 us, 128 x 128 18.4; 1000 x 1000 -> 2 x 4096 (1024) 30.5 and 24.3
//   500 x 512 -> 2 x 1365 (float32): 64 rows 23.7 us, 128 x 128 40.2
//   dX of 512 x 1024, 4096 (bfloat16): 64 rows in four parts 24 us, in eight 23, in one 54, 128 x 128 in eight 24, 256 x 256 163
//   2048 x 4096 -> 2 x 4096 (bfloat16): 256 x 256 107 us, 128 x 128 128
struct Cost { double fixed, alone, two, round; };  // round: of two, where more tiles follow
inline Cost cost_of(const Shape &s, int kind) {
    static const Cost f32[] = {{}, {6, 1.8, 3.6, 3.6}, {5, 1.0, 1.85, 1.85}};
    static const Cost b16[] = {{7, 1.5}, {6, 0.50, 0.97, 0.97}, {5, 0.32, 0.56, 0.65}};
    static const Cost mx4[] = {{7, 1.6}, {6, 0.75, 1.4, 1.4}, {5, 0.50, 0.90, 0.90}};
    Cost c = (s.E == kF32 ? f32 : s.E == kMX4 ? mx4 : b16)[kind];
    if (s.strided && s.E == kF32) {
        if (kind == k128) c.alone *= 1.2;
    } else if (s.strided && kind != kBig) {
        c.alone *= 1.3;
        if (kind == k64) c.round = c.two *= 1.07;
    }
    return c;
}
inline double depth_of(const Shape &s, const Plan &p) { return (double)(long long)(p.ktiles * s.segs / p.splits); }
inline double join_time(const Plan &p) { return p.splits > 1 ? 4 + (double)p.workspace * 2 / 8e6 : 0; }
inline double time_of(const Shape &s, const Plan &p, int cus) {
    const Cost c = cost_of(s, p.kind);
    const long long tiles = (long long)p.tiles_m * p.tiles_n * s.results * p.splits;
    const double depth = depth_of(s, p);
    double t;
    if (p.kind == kBig) {
        t = c.fixed + (double)up(tiles, cus) * (depth * c.alone + 6);
    } else {
        const long long full = tiles / (2 * cus), left = tiles % (2 * cus);
        t = c.fixed + (double)full * (depth * c.round + 2);
        if (left) t += depth * (left <= cus ? c.alone : c.two);
    }
    return t + join_time(p);
}
// (a launch that joins has less than 2^32 threads, of four sums each)
inline bool can_split(const Shape &s, const Plan &p) { return p.ktiles * s.segs >= 2 * p.splits && s.results * s.M * s.N < 1LL << 33; }
// workspace: bytes there are for a split.
inline Plan plan_tiles(const Shape &s, long long workspace, int cus) {
    Plan best{};
    double least = 0;
    for (int kind : {kBig, k128, k64}) {
        if (kind == kBig && s.E == kF32) continue;
        for (int splits : {1, 2, 3, 4, 6, 8, 12, 16}) {
            const Plan p = plan_of(s, kind, splits);
            if (splits > 1 && (kind == kBig || p.workspace > workspace || !can_split(s, p))) break;
            const double t = time_of(s, p, cus);
            if (best.tiles_m == 0 || t < least) { best = p; least = t; }
        }
    }
    return best;
}
inline long long whole256(long long bytes) { return (bytes + 255) / 256 * 256; }

// 128 rows with four K tiles in LDS (k_mid); gradients of such shapes take tiles of 64 rows.
inline bool deep_tiles(int E, bool strided, const Plan &p, int results, int cus) {
    return p.kind == k128 && E != kF32 && !strided && (long long)p.tiles_m * p.tiles_n * results * p.splits <= cus && p.ktiles >= 32 * p.splits;
}

// Both gradients' plans: in one launch where that takes less than one after the other, as it does but for the largest
// tiles.  T x D, F, one after the other and together, with the sums joined: 500 x 512, 1365 (float32) 50 and 40 us;
// 333 x 1000, 2730 (bfloat16) 36 and 30; 256 x 512, 2048 18.4 and 12.6; 2048 x 1024, 4096 78 and 71; 2048 x 4096,
// 4096 237 and 254.
struct Plans {
    Plan x, w;
    bool together;
    long long workspace;
};
inline Plans plan_pair(const Shape &x, const Shape &w, int cus) {
    Plans best{plan_tiles(x, INT64_MAX, cus), plan_tiles(w, INT64_MAX, cus), false, 0};
    const long long apart = std::max(best.x.workspace, best.w.workspace);  // (one of them alone may be asked for)
    best.workspace = apart;
    double least = 0.97 * (time_of(x, best.x, cus) + time_of(w, best.w, cus) + 4);
    for (int kx : {k128, k64}) {
        const Cost cx = cost_of(x, kx);
        for (int sx : {1, 2, 4, 8, 16}) {
            const Plan px = plan_of(x, kx, sx);
            if (sx > 1 && !can_split(x, px)) break;
            const double dx = depth_of(x, px), nx = (double)px.tiles_m * px.tiles_n * sx;
            for (int kw : {k128, k64}) {
                const Cost cw = cost_of(w, kw);
                for (int sw : {1, 2, 4, 8}) {
                    const Plan pw = plan_of(w, kw, sw);
                    if (sw > 1 && !can_split(w, pw)) break;
                    const double dw = depth_of(w, pw), nw = (double)pw.tiles_m * pw.tiles_n * 2 * sw;
                    const bool alone = nx + nw <= cus;
                    const double longx = dx * (alone ? cx.alone : cx.two), longw = dw * (alone ? cw.alone : cw.two);
                    // all the work shared out (a tenth less than of one kind: short workgroups fill what long ones
                    // leave), or the longest workgroup
                    const double shared = 0.9 * (nx * dx * cx.two + nw * dw * cw.two) / 2 / cus + 4 * (nx + nw) / (2 * cus);
                    const double joins = (sx > 1 ? 2 : 0) + (sw > 1 ? 2 : 0) + (double)(px.workspace + pw.workspace) * 2 / 3e6;
                    const double t = 6 + std::max(shared, std::max(longx, longw)) + joins;
                    if (t < least && nx + nw < 1 << 23) {
                        least = t;
                        best = {px, pw, true, std::max(apart, whole256(px.workspace) + pw.workspace)};
                    }
                }
            }
        }
    }
    return best;
}
// A few rows of A: k_few's way is the shortest while the weights are not much (each of its wavefronts waits for its own
// loads; tiles have more of them in flight), and the less so the more rows multiply each of them.  Its workgroups have 16
// columns: many of them start slowly, and few, of long rows, leave compute units idle.  float32 tiles multiply 64 rows at a
// sixteenth of the 16-bit rate however few there are, and odd rows are copied for them first.  In us, k_few and tiles, one set of
// operands over and over (with others in between tiles gain where rows are more than a few: bfloat16, 32 x 2048 -> 2 x 4096 14.8, 12.0;
// 16 x 2048 -> 2 x 8192 20.9, 15.4; 1 row 13.1, 14.9; 64 x 1000 -> 2 x 2728 8.6, 10.9):
//   bfloat16   1 x 2048 -> 2 x 8192 (67 MB) 13.2, 15.1; 16 rows 15.6, 15.4; 16 x 4096 -> 2 x 8192 29.0, 25.5; 32 x 2048 ->
//              2 x 4096 10.8, 11.4; 64 x 2048 -> 2 x 4096 15.1, 13.1; 64 x 1000 -> 2 x 2728 7.1, 9.5;
//              16 x 8192 -> 2 x 2048 23.9, 16.1; 16 x 512 -> 2 x 16384 8.5, 6.8
//   float32    16 x 4096 -> 2 x 8192 58, 74; 32 rows 92, 74; 32 x 2048 -> 2 x 4096 24.7, 25.5; 64 x 2047 -> 2 x 4096 42, 48
//   four bits  1 x 8192 -> 8192 8.9, 11.7; 16384 20.6, 16.6; 16 x 4096 -> 11008 9.2, 13.0; 32 x 8192 -> 8192 22.6, 12.8
inline bool few_rows(int E, int M, int N, int K, bool gated, int cus) {
    static const int f32[] = {540, 68, 20}, b16[] = {68, 34, 12}, mx4[] = {36, 18, 9};  // MB of weights for 16, 32, 64 rows
    if (M > 64) return false;
    const long long row = E == kMX4 ? K / 2 : (long long)K * bytes_of(E);
    const int most = (E == kF32 ? f32 : E == kMX4 ? mx4 : b16)[M <= 16 ? 0 : M <= 32 ? 1 : 2];
    if (E == kF32 && K % per16(E)) return true;  // 64 x 4095 -> 2 x 8191 156, 184
    if (E != kF32 && (row > 8192 || up(N, 16) > (M > 16 ? 1 : E == kMX4 ? 3 : 2) * cus)) return false;
    const bool odd = K % per16(E) != 0;  // 1 x 4095 -> 2 x 8191 (bfloat16) 58, 70; 16 rows 78, 74
    return (gated ? 2 : 1) * row * N <= (odd && M <= 16 ? 2 : 1) * most * 1000000LL;
}

}  // namespace tile
}  // namespace alcs
