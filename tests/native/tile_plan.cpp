// The feed-forward products' choice of kernels (csrc/alcs_tile_plan.h) as C functions, for operands that the tiles take
// or that there is room to copy.
#include "alcs_tile_plan.h"

using namespace alcs::tile;

static void put(int *out, const Shape &s, const Plan &p, int cus) {
    out[0] = p.kind; out[1] = p.splits; out[2] = p.tiles_m * p.tiles_n * s.results; out[3] = p.ktiles * s.segs;
    out[4] = deep_tiles(s.E, s.strided, p, s.results, cus);
}
// kind (3: k_few), parts of K, tiles, K tiles, four K tiles in LDS
extern "C" void linear_plan(int M, int N, int K, long long workspace, int cus, int *out) {
    const Shape s = linear_shape(M, N, K);
    put(out, s, plan_tiles(s, workspace, cus), cus);
    if (few_rows(kMX4, M, N, K, false, cus)) out[0] = 3;
}
extern "C" void forward_plan(int E, int T, int D, int F, long long workspace, int cus, int *out) {
    const Shape s = forward_shape(E, T, whole_pieces(D, E), F);
    put(out, s, plan_tiles(s, workspace, cus), cus);
    if (few_rows(E, T, F, D, true, cus)) out[0] = 3;
}
// out[0]: both gradients in one launch; then dX's plan and dW's; and those of a call that asks for one of them alone
extern "C" void backward_plan(int E, int T, int D, int F, int cus, int *out) {
    const Shape x = dx_shape(E, T, D, whole_pieces(F, E)), w = dw_shape(E, T, D, F);
    const Plans p = plan_pair(x, w, cus);
    out[0] = p.together;
    put(out + 1, x, p.together ? p.x : plan_tiles(x, p.workspace, cus), cus);
    put(out + 6, w, p.together ? p.w : plan_tiles(w, p.workspace, cus), cus);
    put(out + 11, x, plan_tiles(x, p.workspace, cus), cus);
    put(out + 16, w, plan_tiles(w, p.workspace, cus), cus);
}
// microseconds, as the rule has it, of a gated product on tiles of one kind
extern "C" double forward_time(int E, int T, int D, int F, int kind, int splits, int cus) {
    const Shape s = forward_shape(E, T, whole_pieces(D, E), F);
    return time_of(s, plan_of(s, kind, splits), cus);
}
