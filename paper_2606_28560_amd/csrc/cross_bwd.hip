// Gradients of dense attention to states of another length.  With the forward's lse_r,
//
//   p_rj = exp(s_rj - lse_r),  D_r = <dO_r, o_r>,  dS_rj = p_rj (<dO_r, v_j> - D_r),
//   dq_r = tau sum_j dS_rj k_j,  dk_j = tau sum_r dS_rj q_r,  dv_j = sum_r p_rj dO_r,
//
// the sums over r running over every query head (and, for states that the batch shares,
// every batch entry) that reads the key/value head.  The weights are formed again in each
// kernel: dq goes by rows and passes over the states, dk and dv go by the states' rows and
// pass over the queries, so that no sum needs atomics and every order is fixed.
#include "cross_launch.h"

namespace fibattn {

namespace {

template <typename S> constexpr int kStage = sizeof(S) == 2 ? 64 : 32;

__device__ __forceinline__ long long stat_at(const Gradients &a, int b, int h, int t) {
    return (((long long)b * a.H + h) * ((a.T + 31) / 32) + t / 32) * 64 + t % 32;
}

// One stage of the states' rows for the dq of a wave's 32 queries.
template <typename S, int D> struct DqRows {
    Frag<S> q[D / 16], g[D / 16];
    f32x16_t acc[D / 32];
    float lse2, delta;
};

template <typename S, int D>
__device__ __forceinline__ void dq_step(const char *__restrict kt, const char *__restrict vt, int row0, int base,
                                        int len, float scale, DqRows<S, D> &w) {
    typedef Tile<S, D> X;
    const int lane = threadIdx.x & 63, h = lane >> 5;
    f32x16_t s = zero16(), u = zero16();
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
        Frag<S> f;
        X::row_frag(kt, row0 + (lane & 31), ks, h, f);
        s = mma(f, w.q[ks], s);
    }
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
        Frag<S> f;
        X::row_frag(vt, row0 + (lane & 31), ks, h, f);
        u = mma(f, w.g[ks], u);
    }
    if (base + 32 > len) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (base + 8 * (i >> 2) + 4 * h + (i & 3) >= len) s[i] = -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = ex2(fmaf(s[i], scale, -w.lse2)) * (u[i] - w.delta);
#pragma unroll
    for (int a = 0; a < 2; ++a) {
        const Weights<S> p(s, a);
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) {
            Frag<S> f;
            X::operand_t(kt, row0 + 16 * a, dt, f);
            w.acc[dt] = p.add(f, w.acc[dt]);
        }
    }
}

// 128 query rows a workgroup, 32 to a wave; the rows of the states are staged for all four.
// The first piece also leaves lse log2 e and D of its rows for dk and dv.
template <typename S, int D>
__global__ __launch_bounds__(256, sizeof(S) == 4 && D == 128 ? 1 : 2) void cross_dq_kernel(Gradients a, int items) {
    typedef Tile<S, D> X;
    constexpr int NT = kStage<S>, TB = NT * X::kRow;
    __shared__ __attribute__((aligned(16))) char lds[4 * TB];
    const int blk = blockIdx.y * gridDim.x + blockIdx.x;
    if (blk >= items) return;
    const int item = xcd_item(blk, items);
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    const int tile = item % a.row_tiles, piece = item / a.row_tiles % a.dq_pieces,
              prob = item / a.row_tiles / a.dq_pieces;
    const int b0 = prob / a.Hkv, j = prob % a.Hkv;
    const int len = a.lens ? min(max(a.lens[b0], 0), a.S) : a.S;
    const int r0 = 128 * tile + 32 * wv, r = r0 + (lane & 31);
    const bool on = r < a.rows, idle = r0 >= a.rows;
    const int rc = min(r, a.rows - 1), hq = rc / a.T, bb = hq / a.G;
    const int b = b0 + bb, hh = j * a.G + (hq - bb * a.G), t = rc - hq * a.T;
    const long long id = ((long long)b * a.H + hh) * a.T + t;

    DqRows<S, D> w;
    const S *q = (const S *)a.q + b * a.lq.sb + hh * a.lq.sh + t * a.lq.st;
    const S *g = (const S *)a.g + b * a.lg.sb + hh * a.lg.sh + t * a.lg.st;
    const S *o = (const S *)a.o + b * a.lo.sb + hh * a.lo.sh + t * a.lo.st;
    float delta = 0.f;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
        Frag<S> f;
        load_frag(q, ks, h, w.q[ks]);
        load_frag(g, ks, h, w.g[ks]);
        load_frag(o, ks, h, f);
        delta += dot_frag(w.g[ks], f);
    }
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) w.acc[dt] = zero16();
    const float lse = a.lse[id];
    // a row that read nothing has weights of 0
    w.lse2 = lse == -INFINITY ? INFINITY : lse * kLog2e;
    w.delta = half_sum(delta);
    if (piece == 0 && on && h == 0) {
        float *st = a.stats + stat_at(a, b, hh, t);
        st[0] = w.lse2;
        st[32] = w.delta;
        // positions behind the last one of the head count nothing
        if (t == a.T - 1)
            for (int e = t + 1; e & 31; ++e) {
                float *x = a.stats + stat_at(a, b, hh, e);
                x[0] = INFINITY;
                x[32] = 0.f;
            }
    }

    const int n = (len + NT - 1) / NT;
    const int n0 = (int)((long long)n * piece / a.dq_pieces), n1 = (int)((long long)n * (piece + 1) / a.dq_pieces);
    const char *kp = (const char *)((const S *)a.k + b0 * a.lk.sb + j * a.lk.sh);
    const char *vp = (const char *)((const S *)a.v + b0 * a.lv.sb + j * a.lv.sh);
    const long long ks = a.lk.st * (long long)sizeof(S), vs = a.lv.st * (long long)sizeof(S);
    auto fetch = [&](int i) {
        const int row = i * NT;
        char *dst = lds + ((i - n0) & 1) * 2 * TB;
        X::template stage<NT, 4>(dst, kp + row * ks, ks, len - row, wv);
        X::template stage<NT, 4>(dst + TB, vp + row * vs, vs, len - row, wv);
    };
    if (n0 < n1) fetch(n0);
    for (int i = n0; i < n1; ++i) {
        wait_loads<0>();
        __syncthreads();  // this stage has arrived, the one before has been read
        if (i + 1 < n1) fetch(i + 1);
        if (idle) continue;
        const char *kt = lds + ((i - n0) & 1) * 2 * TB;
#pragma unroll
        for (int e = 0; e < NT / 32; ++e)
            if (i * NT + 32 * e < len) dq_step<S, D>(kt, kt + TB, 32 * e, i * NT + 32 * e, len, a.scale, w);
    }
    if (!on) return;
    if (a.dq_pieces > 1) {
        const long long rows = (long long)a.B * a.H * a.T;
        store_cols<D>(a.dq_part + (piece * rows + id) * D, w.acc, a.tau, h);
    } else {
        store_cols<D>((S *)a.dq + b * a.ldq.sb + hh * a.ldq.sh + t * a.ldq.st, w.acc, a.tau, h);
    }
}

// 128 rows of the states a workgroup, 32 to a wave with their k and v in registers; tiles of
// 32 queries of one head (q, dO and their lse, D) are staged for all four, two at a time.
template <typename S, int D>
__global__ __launch_bounds__(256, D == 128 ? 1 : 2) void cross_dkdv_kernel(Gradients a, int items) {
    typedef Tile<S, D> X;
    constexpr int QT = kStage<S> / 32, TB = 32 * X::kRow, SB = 2 * TB + 256;  // q, dO, statistics
    __shared__ __attribute__((aligned(16))) char lds[2 * QT * SB];
    const int blk = blockIdx.y * gridDim.x + blockIdx.x;
    if (blk >= items) return;
    const int item = xcd_item(blk, items);
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    const int tile = item % a.key_tiles, piece = item / a.key_tiles % a.dkv_pieces,
              prob = item / a.key_tiles / a.dkv_pieces;
    const int b0 = prob / a.Hkv, j = prob % a.Hkv;
    const int len = a.lens ? min(max(a.lens[b0], 0), a.S) : a.S;
    const int c0 = 128 * tile + 32 * wv, c = c0 + (lane & 31);

    f32x16_t dk[D / 32], dv[D / 32];
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) dk[dt] = dv[dt] = zero16();
    if (128 * tile < len) {
        Frag<S> kf[D / 16], vf[D / 16];
        const int cc = min(c, len - 1);
        const S *k = (const S *)a.k + b0 * a.lk.sb + j * a.lk.sh + cc * a.lk.st;
        const S *v = (const S *)a.v + b0 * a.lv.sb + j * a.lv.sh + cc * a.lv.st;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
            load_frag(k, ks, h, kf[ks]);
            load_frag(v, ks, h, vf[ks]);
        }
        const int tiles = (a.T + 31) / 32;  // of a head
        const int n = tiles * a.G * a.share;
        const int n0 = (int)((long long)n * piece / a.dkv_pieces),
                  n1 = (int)((long long)n * (piece + 1) / a.dkv_pieces);
        const long long qs = a.lq.st * (long long)sizeof(S), gs = a.lg.st * (long long)sizeof(S);
        auto fetch = [&](int i, int slot) {
            const int hq = i / tiles, t0 = (i - hq * tiles) * 32, bb = hq / a.G;
            const int b = b0 + bb, hh = j * a.G + (hq - bb * a.G);
            char *dst = lds + slot * SB;
            X::template stage<32, 4>(dst, (const char *)((const S *)a.q + b * a.lq.sb + hh * a.lq.sh + t0 * a.lq.st),
                                     qs, a.T - t0, wv);
            X::template stage<32, 4>(dst + TB,
                                     (const char *)((const S *)a.g + b * a.lg.sb + hh * a.lg.sh + t0 * a.lg.st), gs,
                                     a.T - t0, wv);
            if (wv == 3)
                load_lds4(uniform(lds_address(dst + 2 * TB)), buffer_of(a.stats + stat_at(a, b, hh, t0), 256), 4 * lane);
        };
        auto fetch_all = [&](int i, int half) {
#pragma unroll
            for (int e = 0; e < QT; ++e)
                if (i + e < n1) fetch(i + e, half * QT + e);
        };
        if (n0 < n1) fetch_all(n0, 0);
        int half = 0;
        for (int i = n0; i < n1; i += QT, half ^= 1) {
            wait_loads<0>();
            __syncthreads();  // this stage has arrived, the one before has been read
            if (i + QT < n1) fetch_all(i + QT, half ^ 1);
            if (c0 >= len) continue;
#pragma unroll
            for (int e = 0; e < QT; ++e) {
                if (i + e >= n1) break;
                const char *qt = lds + (half * QT + e) * SB, *gt = qt + TB;
                const float *st = (const float *)(qt + 2 * TB);
                f32x16_t s = zero16(), u = zero16();
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    Frag<S> f;
                    X::row_frag(qt, lane & 31, ks, h, f);
                    s = mma(f, kf[ks], s);
                }
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    Frag<S> f;
                    X::row_frag(gt, lane & 31, ks, h, f);
                    u = mma(f, vf[ks], u);
                }
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const f32x4_t lse2 = *reinterpret_cast<const f32x4_t *>(st + 8 * x + 4 * h);
                    const f32x4_t delta = *reinterpret_cast<const f32x4_t *>(st + 32 + 8 * x + 4 * h);
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        const float p = ex2(fmaf(s[4 * x + y], a.scale, -lse2[y]));
                        s[4 * x + y] = p;
                        u[4 * x + y] = p * (u[4 * x + y] - delta[y]);
                    }
                }
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const Weights<S> p(s, x), ds(u, x);
#pragma unroll
                    for (int dt = 0; dt < D / 32; ++dt) {
                        Frag<S> f;
                        X::operand_t(gt, 16 * x, dt, f);
                        dv[dt] = p.add(f, dv[dt]);
                        X::operand_t(qt, 16 * x, dt, f);
                        dk[dt] = ds.add(f, dk[dt]);
                    }
                }
            }
        }
    }
    if (c >= a.S) return;
    if (c >= len) {  // rows that no query reads
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) dk[dt] = dv[dt] = zero16();
    }
    if (a.dkv_pieces > 1) {
        if (c >= len) return;  // the sum over the pieces writes those zeros
        const long long rows = (long long)a.Bkv * a.Hkv * a.S, id = (long long)prob * a.S + c;
        store_cols<D>(a.dk_part + (piece * rows + id) * D, dk, a.tau, h);
        store_cols<D>(a.dv_part + (piece * rows + id) * D, dv, 1.f, h);
    } else {
        store_cols<D>((S *)a.dk + b0 * a.ldk.sb + j * a.ldk.sh + c * a.ldk.st, dk, a.tau, h);
        store_cols<D>((S *)a.dv + b0 * a.ldv.sb + j * a.ldv.sh + c * a.ldv.st, dv, 1.f, h);
    }
}

// Sums the pieces of up to three gradients, in the order of the pieces.
struct SumJob {
    const float *part;
    void *out;
    Layout l;
    const int *lens;  // rows behind them are 0 (null: none)
    long long rows;   // B heads T
    int pieces, heads, T;
};
struct SumJobs {
    SumJob job[3];
};
template <typename S, int D> __global__ __launch_bounds__(256) void sum_pieces_kernel(SumJobs jobs) {
    const SumJob j = jobs.job[blockIdx.z];
    constexpr int per = D / 4;
    const long long e = ((long long)blockIdx.y * gridDim.x + blockIdx.x) * 256 + threadIdx.x, r = e / per;
    if (r >= j.rows) return;
    const int d = (int)(e % per) * 4;
    const int t = (int)(r % j.T), h = (int)(r / j.T % j.heads), b = (int)(r / j.T / j.heads);
    f32x4_t y = {0.f, 0.f, 0.f, 0.f};
    if (!j.lens || t < j.lens[b])
        for (int i = 0; i < j.pieces; ++i) y += *reinterpret_cast<const f32x4_t *>(j.part + (i * j.rows + r) * D + d);
    S *row = (S *)j.out + b * j.l.sb + h * j.l.sh + t * j.l.st + d;
    if constexpr (sizeof(S) == 4)
        *reinterpret_cast<f32x4_t *>(row) = y;
    else
        *reinterpret_cast<uint2 *>(row) = make_uint2(pack2(y[0], y[1]), pack2(y[2], y[3]));
}

template <typename S, int D> hipError_t backward(Gradients a, hipStream_t st) {
    const int prob = a.Bkv * a.Hkv;
    const long long n = (long long)prob * a.row_tiles * a.dq_pieces, m = (long long)prob * a.key_tiles * a.dkv_pieces;
    if (n >= 1ll << 31 || m >= 1ll << 31) return hipErrorInvalidValue;
    hipError_t e = launch(kCrossBwdDq, cross_dq_kernel<S, D>, grid_of(n), dim3(256), 0, st, a, (int)n);
    if (e != hipSuccess) return e;
    e = launch(kCrossBwdDkDv, cross_dkdv_kernel<S, D>, grid_of(m), dim3(256), 0, st, a, (int)m);
    if (e != hipSuccess) return e;
    SumJobs jobs{};
    int count = 0;
    long long most = 0;
    if (a.dq_pieces > 1) {
        jobs.job[count++] = {a.dq_part, a.dq, a.ldq, nullptr, (long long)a.B * a.H * a.T, a.dq_pieces, a.H, a.T};
        most = (long long)a.B * a.H * a.T;
    }
    if (a.dkv_pieces > 1) {
        const long long rows = (long long)prob * a.S;
        jobs.job[count++] = {a.dk_part, a.dk, a.ldk, a.lens, rows, a.dkv_pieces, a.Hkv, a.S};
        jobs.job[count++] = {a.dv_part, a.dv, a.ldv, a.lens, rows, a.dkv_pieces, a.Hkv, a.S};
        most = most > rows ? most : rows;
    }
    if (!count) return hipSuccess;
    dim3 grid = grid_of((most * (D / 4) + 255) / 256);
    grid.z = count;
    return launch(kJoin, sum_pieces_kernel<S, D>, grid, dim3(256), 0, st, jobs);
}

template <typename S> hipError_t backward_d(int D, const Gradients &a, hipStream_t s) {
    switch (D) {
        case 32: return backward<S, 32>(a, s);
        case 64: return backward<S, 64>(a, s);
        default: return backward<S, 128>(a, s);
    }
}

// Pieces of a sum: enough for two workgroups to a CU, `least` rows or more to each.
int pieces(long long wgs, long long steps, int least) {
    const long long want = (512 + wgs - 1) / wgs, most = (steps + least - 1) / least;
    const long long n = want < most ? want : most;
    return (int)(n < 1 ? 1 : n > 64 ? 64 : n);
}

}  // namespace

void plan_cross_backward(Gradients *a) {
    const long long prob = (long long)a->Bkv * a->Hkv;
    a->row_tiles = (a->rows + 127) / 128;
    a->key_tiles = (a->S + 127) / 128;
    a->dq_pieces = pieces(prob * a->row_tiles, a->S, 512);
    a->dkv_pieces = pieces(prob * a->key_tiles, a->rows, 512);
}

hipError_t launch_cross_backward(int dtype, int D, const Gradients &a, hipStream_t s) {
    return dtype == 1 ? backward_d<uint16_t>(D, a, s) : backward_d<float>(D, a, s);
}

}  // namespace fibattn
