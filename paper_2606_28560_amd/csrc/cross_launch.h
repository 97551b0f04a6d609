// Host-side launchers of the kernels for attention to other states (cross_fwd.hip,
// cross_bwd.hip).
#pragma once

#include "cross.h"
#include "launch.h"

namespace fibattn {

// How the forward reads the states (rw, tiles, splits, slot, from their rows and S); the partial
// results it makes of each row.  s1: null, or the second states.
int plan_cross_forward(int dtype, int D, States *s0, States *s1, int prob0, int prob1);

// Attention to s0 and, when s1 is not null, to s1 too, in one softmax, as planned; prob0, prob1:
// their problems.  a.part_o and a.part_lse are read and written only where the pieces of both are
// more than one.
hipError_t launch_cross_forward(int dtype, int D, const Queries &a, const States &s0, const States *s1, int prob0,
                                int prob1, hipStream_t s);

struct JoinArgs {
    const void *a, *b;
    const float *za, *zb;
    void *o;
    float *z;
    Layout la, lb, lo;
    int B, H, T;
};
hipError_t launch_join(int dtype, int D, const JoinArgs &a, hipStream_t s);

// The gradients of attention to one set of states (cross_bwd.hip).
struct Gradients {
    const void *q, *k, *v, *o, *g;
    const float *lse;
    void *dq, *dk, *dv;
    Layout lq, lk, lv, lo, lg, ldq, ldk, ldv;
    const int *lens;
    float *stats;  // per tile of 32 positions of a head: lse log2 e of each, then -<dO, o>
    float *dq_part, *dk_part, *dv_part;  // [piece][rows][D] where a sum is made in pieces
    int B, Bkv, H, Hkv, G, T, S, share, rows;  // share: B where Bkv is 1, else 1; rows: share G T
    int row_tiles, key_tiles, dq_pieces, dkv_pieces, dq_narrow, dkv_narrow;
    float scale, tau;  // tau log2 e, tau
};
void plan_cross_backward(int dtype, int D, Gradients *a);  // the tiles and pieces, from the sizes
hipError_t launch_cross_backward(int dtype, int D, const Gradients &a, hipStream_t s);

}  // namespace fibattn
