// Gradients of dense attention to states of another length.  With the forward's lse_r,
//
//   p_rj = exp(s_rj - lse_r),  D_r = <dO_r, o_r>,  dS_rj = p_rj (<dO_r, v_j> - D_r),
//   dq_r = tau sum_j dS_rj k_j,  dk_j = tau sum_r dS_rj q_r,  dv_j = sum_r p_rj dO_r,
//
// D from the o that was stored, whose rounding it has (2^-8 of its terms in bfloat16): its other
// form, sum_j p_rj <dO_r, v_j>, holds only where these states are the whole softmax, and needs
// a pass over them before dq's.  Of lse_r and o_r those of a softmax over more keys do as well.
//
// the sums over r running over every query head (and, for states that the batch shares,
// every batch entry) that reads the key/value head.  The weights are formed again in each
// kernel: dq goes by rows and passes over the states, dk and dv go by the states' rows and
// pass over the queries, so that no sum needs atomics and every order is fixed.
#include "cross_launch.h"

namespace fibattn {

namespace {

// Rows of the states that the wide dq kernel stages at a time.
template <typename S> constexpr int kStage = sizeof(S) == 2 ? 64 : 32;

__device__ __forceinline__ long long stat_at(const Gradients &a, int b, int h, int t) {
    return (((long long)b * a.H + h) * ((a.T + 31) / 32) + t / 32) * 64 + t % 32;
}

// A wave's 32 query rows: q, dO, lse log2 e, -<dO, o>, and their dq.
template <typename S, int D> struct DqRows {
    Frag<S> q[D / 16], g[D / 16];
    f32x16_t acc[D / 32];
    float lse2, delta;
};

// s = q k and u = dO v of 32 staged rows of the states.
template <typename S, int D>
__device__ __forceinline__ void dq_products(const char *kt, const char *vt, int row0, f32x16_t &s, f32x16_t &u,
                                            const DqRows<S, D> &w) {
    typedef Tile<S, D> X;
    const int lane = threadIdx.x & 63, h = lane >> 5;
    s = u = zero16();
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
}
// dq += dS k over them; their first is row `base` of len.
template <typename S, int D>
__device__ __forceinline__ void dq_add(const char *kt, int row0, int base, int len, float scale, f32x16_t &s,
                                       const f32x16_t &u, DqRows<S, D> &w) {
    const int h = (threadIdx.x >> 5) & 1;
    if (base + 32 > len) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (base + 8 * (i >> 2) + 4 * h + (i & 3) >= len) s[i] = -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = ex2(fmaf(s[i], scale, -w.lse2)) * (u[i] + w.delta);
#pragma unroll
    for (int a = 0; a < 2; ++a) {
        const Weights<S> p(s, a);
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) {
            Frag<S> f;
            Tile<S, D>::operand_t(kt, row0 + 16 * a, dt, f);
            w.acc[dt] = p.add(f, w.acc[dt]);
        }
    }
}

// What the products of dk and dv take their operands from.
template <typename S, int D> struct KvValue { typedef S type; };
template <> struct KvValue<float, 128> { typedef whole_t type; };

// 32 rows of the states of a wave, and their gradients (S: a KvValue).
template <typename S, int D> struct KvRows {
    Frag<S> k[D / 16], v[D / 16];
    f32x16_t dk[D / 32], dv[D / 32];
};

// The weights p (in s) and dS (in u) of a staged tile of queries: q, dO, statistics.
// The sum of dO v begins at -<dO, o>, read where it accumulates: 16 subtractions less a tile
// (57.3 for 58.5 microseconds at 8 x 8 heads of 1024 x 1024, d 64, bfloat16; 115 for 127 at
// 4 x 8 of 1000 x 1000 in float32).  In dq, which has one value of it to a lane, the copies that
// 16 accumulators would begin with took as long as the subtractions.
template <typename S, int D>
__device__ __forceinline__ void kv_products(const char *qt, float scale, f32x16_t &s, f32x16_t &u,
                                            const KvRows<S, D> &w) {
    typedef Tile<S, D> X;
    const int lane = threadIdx.x & 63, h = lane >> 5;
    const char *gt = qt + X::bytes(32);
    const float *st = (const float *)(gt + X::bytes(32));
    s = zero16();
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        const f32x4_t delta = *reinterpret_cast<const f32x4_t *>(st + 32 + 8 * x + 4 * h);  // -<dO, o>
#pragma unroll
        for (int y = 0; y < 4; ++y) u[4 * x + y] = delta[y];
    }
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
        Frag<S> f;
        X::row_frag(qt, lane & 31, ks, h, f);
        s = mma(f, w.k[ks], s);
    }
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
        Frag<S> f;
        X::row_frag(gt, lane & 31, ks, h, f);
        u = mma(f, w.v[ks], u);
    }
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        const f32x4_t lse2 = *reinterpret_cast<const f32x4_t *>(st + 8 * x + 4 * h);
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            const float p = ex2(fmaf(s[4 * x + y], scale, -lse2[y]));
            s[4 * x + y] = p;
            u[4 * x + y] *= p;
        }
    }
}
// dv += p dO and dk += dS q over the tile.  A wave's matrix instructions go before the other
// waves' exponentials (s_setprio): 65 to 60 microseconds at 8 x 8 heads of 1024 x 1024, d 64;
// in the forward and dq, whose runs of them are shorter, it changed nothing.
template <typename S, int D>
__device__ __forceinline__ void kv_add_v(const char *qt, const f32x16_t &p, KvRows<S, D> &w) {
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const Weights<S> pw(p, x);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) {
            Frag<S> f;
            Tile<S, D>::operand_t(qt + Tile<S, D>::bytes(32), 16 * x, dt, f);
            w.dv[dt] = pw.add(f, w.dv[dt]);
        }
        __builtin_amdgcn_s_setprio(0);
    }
}
template <typename S, int D>
__device__ __forceinline__ void kv_add_k(const char *qt, const f32x16_t &ds, KvRows<S, D> &w) {
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const Weights<S> dw(ds, x);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) {
            Frag<S> f;
            Tile<S, D>::operand_t(qt, 16 * x, dt, f);
            w.dk[dt] = dw.add(f, w.dk[dt]);
        }
        __builtin_amdgcn_s_setprio(0);
    }
}

// One item of the dq kernels: its problem, its rows and its piece of the states.
template <typename S, int D> struct DqItem {
    int b0, j, piece, len;
    const char *kp, *vp;
    long long ks, vs;
    int b, hh, t;  // the lane's row
    long long id;
    bool on;

    __device__ __forceinline__ DqItem(const Gradients &a, int prob, int row0, int piece_) {
        b0 = prob / a.Hkv;
        j = prob % a.Hkv;
        piece = piece_;
        len = a.lens ? min(max(a.lens[b0], 0), a.S) : a.S;
        kp = (const char *)((const S *)a.k + b0 * a.lk.sb + j * a.lk.sh);
        vp = (const char *)((const S *)a.v + b0 * a.lv.sb + j * a.lv.sh);
        ks = a.lk.st * (long long)sizeof(S);
        vs = a.lv.st * (long long)sizeof(S);
        const int r = row0 + (int)(threadIdx.x & 31), rc = min(r, a.rows - 1), hq = rc / a.T, bb = hq / a.G;
        on = r < a.rows;
        b = b0 + bb;
        hh = j * a.G + (hq - bb * a.G);
        t = rc - hq * a.T;
        id = ((long long)b * a.H + hh) * a.T + t;
    }
    // The rows' q, dO, lse and D; the first piece leaves lse log2 e and D for dk and dv.
    __device__ __forceinline__ void load(const Gradients &a, bool leave, DqRows<S, D> &w) const {
        const int h = (threadIdx.x >> 5) & 1;
        const S *q = (const S *)a.q + b * a.lq.sb + hh * a.lq.sh + t * a.lq.st;
        const S *g = (const S *)a.g + b * a.lg.sb + hh * a.lg.sh + t * a.lg.st;
        const S *o = (const S *)a.o + b * a.lo.sb + hh * a.lo.sh + t * a.lo.st;
        float delta = 0.f;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
            load_frag(q, ks, h, w.q[ks]);
            load_frag(g, ks, h, w.g[ks]);
            delta += dot_rows(g, o, ks, h);
        }
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) w.acc[dt] = zero16();
        const float lse = a.lse[id];
        // a row that read nothing has weights of 0
        w.lse2 = lse == -INFINITY ? INFINITY : lse * kLog2e;
        w.delta = -half_sum(delta);
        if (leave && on && h == 0) {
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
    }
    // Columns 32 dt .. of the lane's row of dq, or of its piece, unless it is one of `skip`.
    template <int N>
    __device__ __forceinline__ void store(const Gradients &a, int d, const f32x16_t *acc, uint32_t skip) const {
        const int h = (threadIdx.x >> 5) & 1;
        if (!on || (skip >> (threadIdx.x & 31) & 1)) return;
        if (a.dq_pieces > 1)
            store_cols<N>(a.dq_part + (piece * ((long long)a.B * a.H * a.T) + id) * D + d, acc, a.tau, h);
        else
            store_cols<N>((S *)a.dq + b * a.ldq.sb + hh * a.ldq.sh + t * a.ldq.st + d, acc, a.tau, h);
    }
};

// Rows of `which` (bit i: the row of lane i) of an item of dq, by the whole wave: a lane to each
// of 64 rows of the states [c0, c1) for the weights, a lane to each value for the sum.
//
// An infinity in a row of the states makes NaN of its float32 products (the parts of a value), of
// the row's weight and so of every value of dq.  Here a weight of 0 is 0, and what is not finite
// stays where the formula has it, in the elements that are infinite themselves.
template <typename S, int D>
__device__ __forceinline__ void plain_dq(const Gradients &a, const DqItem<S, D> &x, const DqRows<S, D> &w, uint32_t which,
                                         int c0, int c1) {
    constexpr int N = (D + 63) / 64;
    const int lane = threadIdx.x & 63;
    const S *k = (const S *)x.kp, *v = (const S *)x.vp;
    for (; which; which &= which - 1) {
        const int i = __builtin_ctz(which);
        const int b = __shfl(x.b, i, 64), hh = __shfl(x.hh, i, 64), t = __shfl(x.t, i, 64);
        const float lse2 = __shfl(w.lse2, i, 64), delta = __shfl(w.delta, i, 64);
        const S *q = (const S *)a.q + b * a.lq.sb + hh * a.lq.sh + t * a.lq.st;
        const S *g = (const S *)a.g + b * a.lg.sb + hh * a.lg.sh + t * a.lg.st;
        float y[N];
#pragma unroll
        for (int n = 0; n < N; ++n) y[n] = 0.f;
        for (int c = c0; c < c1; c += 64) {
            float ds = 0.f;
            if (c + lane < c1) {
                const float s = dot_row<S, D>(q, k + (c + lane) * a.lk.st);
                ds = ex2(fmaf(s, a.scale, -lse2)) * (dot_row<S, D>(g, v + (c + lane) * a.lv.st) + delta);
            }
            const int count = min(64, c1 - c);
            for (int e = 0; e < count; ++e) {
                const float d = __shfl(ds, e, 64);
#pragma unroll
                for (int n = 0; n < N; ++n)
                    if (lane + 64 * n < D) y[n] = fmaf(d, value_of(k[(c + e) * a.lk.st + lane + 64 * n]), y[n]);
            }
        }
        const long long id = ((long long)b * a.H + hh) * a.T + t;
#pragma unroll
        for (int n = 0; n < N; ++n)
            if (lane + 64 * n < D) {
                if (a.dq_pieces > 1)
                    a.dq_part[(x.piece * ((long long)a.B * a.H * a.T) + id) * D + lane + 64 * n] = y[n] * a.tau;
                else
                    put_value((S *)a.dq + b * a.ldq.sb + hh * a.ldq.sh + t * a.ldq.st + lane + 64 * n, y[n] * a.tau);
            }
    }
}

// Rows that plain_dq does (bit i: the row of lane i), from any value of the lane's row: float32
// rows that are not a number though their lse and D are finite (a weight that is none makes all
// of a row so).
template <typename S, int D>
__device__ __forceinline__ uint32_t odd_rows(const DqItem<S, D> &x, const DqRows<S, D> &w, float any) {
    if constexpr (sizeof(S) == 2) return 0;
    const unsigned long long bad =
        __ballot(x.on && any != any && fabsf(w.lse2) < INFINITY && fabsf(w.delta) < INFINITY);
    return (uint32_t)(bad | bad >> 32);
}

// 128 query rows a workgroup, 32 to a wave; the rows of the states are staged for all four.
template <typename S, int D>
__global__ __launch_bounds__(256, sizeof(S) == 4 && D == 128 ? 1 : 2) void cross_dq_kernel(Gradients a, int items) {
    typedef Tile<S, D> X;
    constexpr int NT = kStage<S>, TB = X::bytes(NT);
    __shared__ __attribute__((aligned(16))) char lds[4 * TB];
    const int blk = blockIdx.y * gridDim.x + blockIdx.x;
    if (blk >= items) return;
    const int item = xcd_item(blk, items);
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tile = item % a.row_tiles, piece = item / a.row_tiles % a.dq_pieces;
    const DqItem<S, D> x(a, item / a.row_tiles / a.dq_pieces, 128 * tile + 32 * wv, piece);
    const bool idle = 128 * tile + 32 * wv >= a.rows;
    const int len = x.len;
    DqRows<S, D> w;

    const int n = (len + NT - 1) / NT;
    const int n0 = (int)((long long)n * piece / a.dq_pieces), n1 = (int)((long long)n * (piece + 1) / a.dq_pieces);
    auto fetch = [&](int i, int half) {
        const int row = i * NT;
        char *dst = lds + half * 2 * TB;
        X::template stage<NT, 4>(dst, x.kp + row * x.ks, x.ks, len - row, wv);
        X::template stage<NT, 4>(dst + TB, x.vp + row * x.vs, x.vs, len - row, wv);
    };
    if (n0 < n1) fetch(n0, 0);
    x.load(a, piece == 0, w);
    wait_loads<0>();  // the queries too: no wait for them stays in the loop
    // one stage from half `half` of the LDS; two to a turn of the loop, so that their addresses
    // are constants (-1 to -2 %)
    auto step = [&](int i, int half) {
        wait_loads<0>();
        __syncthreads();  // this stage has arrived, the one before has been read
        if (i + 1 < n1) fetch(i + 1, half ^ 1);
        if (idle) return;
        const char *kt = lds + half * 2 * TB;
#pragma unroll
        for (int e = 0; e < NT / 32; ++e)
            if (i * NT + 32 * e < len) {
                f32x16_t s, u;
                dq_products<S, D>(kt, kt + TB, 32 * e, s, u, w);
                dq_add<S, D>(kt, 32 * e, i * NT + 32 * e, len, a.scale, s, u, w);
            }
    };
    for (int i = n0; i < n1; i += 2) {
        step(i, 0);
        if (i + 1 < n1) step(i + 1, 1);
    }
    const uint32_t odd = odd_rows<S, D>(x, w, w.acc[0][0]);
    x.template store<D>(a, 0, w.acc, odd);
    if (odd) plain_dq<S, D>(a, x, w, odd, n0 * NT, min(n1 * NT, len));
}

// The four waves' results of the same columns, added in the order of the waves: wave w hands
// tiles w, w + 4, .. to `put`.  `lds` holds 4 KB to a wave and tile.
template <int N, typename Put>
__device__ __forceinline__ void add_waves(const f32x16_t *acc, char *lds, int wv, Put put) {
    const int lane = threadIdx.x & 63;
    float *x = (float *)lds;
    __syncthreads();
#pragma unroll
    for (int dt = 0; dt < N; ++dt)
#pragma unroll
        for (int e = 0; e < 16; e += 4)
            *reinterpret_cast<f32x4_t *>(x + ((wv * N + dt) * 4 + e / 4) * 256 + 4 * lane) =
                f32x4_t{acc[dt][e], acc[dt][e + 1], acc[dt][e + 2], acc[dt][e + 3]};
    __syncthreads();
    for (int dt = wv; dt < N; dt += 4) {
        f32x16_t sum = zero16();
#pragma unroll
        for (int o = 0; o < 4; ++o)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const f32x4_t y = *reinterpret_cast<const f32x4_t *>(x + ((o * N + dt) * 4 + e / 4) * 256 + 4 * lane);
#pragma unroll
                for (int z = 0; z < 4; ++z) sum[e + z] += y[z];
            }
        put(dt, sum);
    }
}

// Every N-th of 32 bits, from bit wv on (N 1, 2 or 4).
template <int N> __device__ __forceinline__ uint32_t every(int wv) {
    return (N == 1 ? 0xffffffffu : N == 2 ? 0x55555555u : 0x11111111u) << wv;
}

// Stages of a wave's own: two where a tile's products are shorter than its way from memory
// (bfloat16), one in float32, whose tiles take twice the LDS and more than twice the time.
template <typename S> constexpr int kPrivate = sizeof(S) == 2 ? 2 : 1;

// 32 query rows for all four waves, each on its own rows of the states (tiles of 32, one in
// four), staged for the wave alone: for problems too few to fill the CUs by 128 rows.
template <typename S, int D>
__global__ __launch_bounds__(256, D == 128 ? 1 : 2) void cross_dq_narrow_kernel(Gradients a, int items) {
    typedef Tile<S, D> X;
    constexpr int NB = kPrivate<S>, TB = X::bytes(32), N = D / 32;
    __shared__ __attribute__((aligned(16))) char lds[8 * NB * TB > 16384 * N ? 8 * NB * TB : 16384 * N];
    const int blk = blockIdx.y * gridDim.x + blockIdx.x;
    if (blk >= items) return;
    const int item = xcd_item(blk, items);
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tile = item % a.row_tiles, piece = item / a.row_tiles % a.dq_pieces;
    const DqItem<S, D> x(a, item / a.row_tiles / a.dq_pieces, 32 * tile, piece);
    const int len = x.len;
    DqRows<S, D> w;

    const int n = (len + 31) / 32;
    const int n0 = (int)((long long)n * piece / a.dq_pieces), n1 = (int)((long long)n * (piece + 1) / a.dq_pieces);
    char *mine = lds + 2 * NB * TB * wv;
    auto fetch_k = [&](int i, char *kt) { X::template stage<32, 1>(kt, x.kp + 32 * i * x.ks, x.ks, len - 32 * i, 0); };
    auto fetch_v = [&](int i, char *kt) {
        X::template stage<32, 1>(kt + TB, x.vp + 32 * i * x.vs, x.vs, len - 32 * i, 0);
    };
    int i = n0 + wv, buf = 0;
    if (i < n1) {
        fetch_v(i, mine);
        fetch_k(i, mine);
    }
    x.load(a, piece == 0 && wv == 0, w);
    wait_loads<0>();  // the queries too: no wait for them stays in the loop
    for (; i < n1; i += 4, buf ^= NB - 1) {
        const bool more = i + 4 < n1;
        char *kt = mine + 2 * TB * buf, *next = mine + 2 * TB * (buf ^ (NB - 1));
        wait_loads<0>();
        wait_lds();
        if (NB == 2 && more) {
            fetch_v(i + 4, next);
            fetch_k(i + 4, next);
        }
        f32x16_t s, u;
        dq_products<S, D>(kt, kt + TB, 0, s, u, w);
        if (NB == 1 && more) {
            wait_lds();  // V has been read
            fetch_v(i + 4, kt);
        }
        dq_add<S, D>(kt, 0, 32 * i, len, a.scale, s, u, w);
        if (NB == 1 && more) {
            wait_lds();  // K has been read
            fetch_k(i + 4, kt);
        }
    }
    uint32_t odd = 0;  // known to the first N waves, which do every N-th of them
    add_waves<N>(w.acc, lds, wv, [&](int dt, const f32x16_t &sum) {
        odd = odd_rows<S, D>(x, w, sum[0]);
        x.template store<32>(a, 32 * dt, &sum, odd);
    });
    odd &= every<N>(wv);
    if (odd) plain_dq<S, D>(a, x, w, odd, 32 * n0, min(32 * n1, len));
}

// One item of the dk, dv kernels: its problem, its piece of the queries, the lane's row of the
// states.
template <typename S, int D> struct KvItem {
    int b0, j, prob, piece, len, c, tiles, n0, n1;
    __device__ __forceinline__ KvItem(const Gradients &a, int prob_, int row0, int piece_) {
        prob = prob_;
        piece = piece_;
        b0 = prob / a.Hkv;
        j = prob % a.Hkv;
        len = a.lens ? min(max(a.lens[b0], 0), a.S) : a.S;
        c = row0 + (int)(threadIdx.x & 31);
        tiles = (a.T + 31) / 32;  // of a query head
        const int n = tiles * a.G * a.share;
        n0 = (int)((long long)n * piece / a.dkv_pieces);
        n1 = (int)((long long)n * (piece + 1) / a.dkv_pieces);
    }
    __device__ __forceinline__ const S *row(const Gradients &a, const void *p, const Layout &l, int cc) const {
        return (const S *)p + b0 * l.sb + j * l.sh + cc * l.st;
    }
    __device__ __forceinline__ void load(const Gradients &a, KvRows<typename KvValue<S, D>::type, D> &w) const {
        const int h = (threadIdx.x >> 5) & 1, cc = min(c, len - 1);
        const S *k = row(a, a.k, a.lk, cc), *v = row(a, a.v, a.lv, cc);
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
            load_frag(k, ks, h, w.k[ks]);
            load_frag(v, ks, h, w.v[ks]);
        }
    }
    // A tile of queries: positions 32 tt .. of member g of the group, batch entry b0 + bb.
    struct At {
        int tt, g, bb;
    };
    __device__ __forceinline__ At tile_at(const Gradients &a, int i) const {
        const int hq = i / tiles, bb = hq / a.G;
        return {i - hq * tiles, hq - bb * a.G, bb};
    }
    __device__ __forceinline__ void step(const Gradients &a, At &at, int by) const {
        at.tt += by;
        while (at.tt >= tiles) {
            at.tt -= tiles;
            if (++at.g == a.G) {
                at.g = 0;
                ++at.bb;
            }
        }
    }
    // Its dO, and its q and statistics, to a stage (q, dO, statistics) by NW waves of which this
    // is w.
    template <int NW> __device__ __forceinline__ void fetch_g(const Gradients &a, const At &at, char *dst, int w) const {
        typedef Tile<S, D> X;
        const S *g = (const S *)a.g + (b0 + at.bb) * a.lg.sb + (j * a.G + at.g) * a.lg.sh + 32 * at.tt * a.lg.st;
        X::template stage<32, NW, true>(dst + X::bytes(32), (const char *)g, a.lg.st * (long long)sizeof(S), a.T - 32 * at.tt, w);
    }
    template <int NW> __device__ __forceinline__ void fetch_q(const Gradients &a, const At &at, char *dst, int w) const {
        typedef Tile<S, D> X;
        const int b = b0 + at.bb, hh = j * a.G + at.g;
        const S *q = (const S *)a.q + b * a.lq.sb + hh * a.lq.sh + 32 * at.tt * a.lq.st;
        X::template stage<32, NW, true>(dst, (const char *)q, a.lq.st * (long long)sizeof(S), a.T - 32 * at.tt, w);
        if (w == NW - 1)
            load_lds4(uniform(lds_address(dst + 2 * X::bytes(32))),
                      buffer_of(a.stats + (((long long)b * a.H + hh) * tiles + at.tt) * 64, 256),
                      4 * (int)(threadIdx.x & 63));
    }
    // Columns d .. d + N - 1 of the lane's row of dk (which 0) or dv (1), or of its piece, unless it
    // is one of `skip`.
    template <int N>
    __device__ __forceinline__ void store(const Gradients &a, int which, int d, const f32x16_t *acc, float scale,
                                          uint32_t skip) const {
        const int h = (threadIdx.x >> 5) & 1;
        if (c >= a.S || (skip >> (threadIdx.x & 31) & 1)) return;
        const f32x16_t none[N / 32] = {};
        const f32x16_t *x = c < len ? acc : none;  // 0 for rows that no query reads
        if (a.dkv_pieces > 1) {
            const long long row = piece * ((long long)a.Bkv * a.Hkv * a.S) + (long long)prob * a.S + c;
            store_cols<N>((which ? a.dv_part : a.dk_part) + row * D + d, x, scale, h);
        } else {
            const Layout &l = which ? a.ldv : a.ldk;
            store_cols<N>((S *)(which ? a.dv : a.dk) + b0 * l.sb + j * l.sh + c * l.st + d, x, scale, h);
        }
    }
    // Rows that plain() does (bit i: the row of lane i), from any value of the lane's row of dk or dv:
    // those that are not a number and whose key holds an infinity (in bfloat16's range) but no NaN.
    // An infinity has no parts: where a product takes them its logits are NaN, and all of dk and dv,
    // though they may be -inf and their weights 0.
    __device__ __forceinline__ uint32_t odd(const Gradients &a, float any) const {
        if constexpr (sizeof(S) == 2 || D == 128) return 0;  // (float32 d 128 multiplies whole values)
        if (!__ballot(c < len && any != any)) return 0;
        const S *k = row(a, a.k, a.lk, min(c, len - 1));
        float top = 0.f, sum = 0.f;
        for (int d = 0; d < D; ++d) {
            const float x = fabsf(value_of(k[d]));
            top = fmaxf(top, x);
            sum += x;
        }
        return (uint32_t)__ballot(c < len && any != any && top >= 0x1.ffp127f && sum == sum);
    }
    // The rows of `which`, each by the whole wave: a lane to each of a tile's queries for the weights,
    // a lane to each value for the sums.
    __device__ __forceinline__ void plain(const Gradients &a, uint32_t which) const {
        constexpr int N = (D + 63) / 64;
        const int lane = threadIdx.x & 63, row0 = __builtin_amdgcn_readfirstlane(c);
        for (; which; which &= which - 1) {
            const int cc = row0 + __builtin_ctz(which);
            const S *k = row(a, a.k, a.lk, cc), *v = row(a, a.v, a.lv, cc);
            float dk[N], dv[N];
#pragma unroll
            for (int n = 0; n < N; ++n) dk[n] = dv[n] = 0.f;
            auto at = tile_at(a, n0);
            for (int i = n0; i < n1; ++i) {
                const int b = b0 + at.bb, hh = j * a.G + at.g, count = min(32, a.T - 32 * at.tt);
                const S *q = (const S *)a.q + b * a.lq.sb + hh * a.lq.sh + 32 * at.tt * a.lq.st;
                const S *g = (const S *)a.g + b * a.lg.sb + hh * a.lg.sh + 32 * at.tt * a.lg.st;
                const float *st = a.stats + (((long long)b * a.H + hh) * tiles + at.tt) * 64;
                float p = 0.f, ds = 0.f;
                if (lane < count) {
                    p = ex2(fmaf(dot_row<S, D>(q + lane * a.lq.st, k), a.scale, -st[lane]));
                    ds = p * (dot_row<S, D>(g + lane * a.lg.st, v) + st[32 + lane]);
                }
                for (int e = 0; e < count; ++e) {
                    const float pe = __shfl(p, e, 64), de = __shfl(ds, e, 64);
#pragma unroll
                    for (int n = 0; n < N; ++n)
                        if (lane + 64 * n < D) {
                            dk[n] = fmaf(de, value_of(q[e * a.lq.st + lane + 64 * n]), dk[n]);
                            dv[n] = fmaf(pe, value_of(g[e * a.lg.st + lane + 64 * n]), dv[n]);
                        }
                }
                step(a, at, 1);
            }
            const long long part = (piece * ((long long)a.Bkv * a.Hkv * a.S) + (long long)prob * a.S + cc) * D;
#pragma unroll
            for (int n = 0; n < N; ++n)
                if (lane + 64 * n < D) {
                    const int d = lane + 64 * n;
                    if (a.dkv_pieces > 1) {
                        a.dk_part[part + d] = dk[n] * a.tau;
                        a.dv_part[part + d] = dv[n];
                    } else {
                        put_value((S *)a.dk + b0 * a.ldk.sb + j * a.ldk.sh + cc * a.ldk.st + d, dk[n] * a.tau);
                        put_value((S *)a.dv + b0 * a.ldv.sb + j * a.ldv.sh + cc * a.ldv.st + d, dv[n]);
                    }
                }
        }
    }
};

// 128 rows of the states a workgroup, 32 to a wave with their k and v in registers; tiles of
// 32 queries of one head (q, dO and their statistics) are staged for all four.
template <typename S, int D>
__global__ __launch_bounds__(256, sizeof(S) == 4 && D == 128 ? 1 : 2) void cross_dkdv_kernel(Gradients a, int items) {
    constexpr int SB = 2 * Tile<S, D>::bytes(32) + 256;
    __shared__ __attribute__((aligned(16))) char lds[2 * SB];
    const int blk = blockIdx.y * gridDim.x + blockIdx.x;
    if (blk >= items) return;
    const int item = xcd_item(blk, items);
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tile = item % a.key_tiles, piece = item / a.key_tiles % a.dkv_pieces;
    const KvItem<S, D> x(a, item / a.key_tiles / a.dkv_pieces, 128 * tile + 32 * wv, piece);
    const bool idle = 128 * tile + 32 * wv >= x.len;
    typedef typename KvValue<S, D>::type V;
    KvRows<V, D> w;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) w.dk[dt] = w.dv[dt] = zero16();
    if (128 * tile < x.len) {
        auto at = x.tile_at(a, x.n0);  // of the tile that is fetched
        auto fetch = [&](int half) {
            x.template fetch_g<4>(a, at, lds + half * SB, wv);
            x.template fetch_q<4>(a, at, lds + half * SB, wv);
            x.step(a, at, 1);
        };
        if (x.n0 < x.n1) fetch(0);
        x.load(a, w);
        wait_loads<0>();  // k and v too: no wait for them stays in the loop
        // one stage, as in dq
        auto step = [&](int i, int half) {
            wait_loads<0>();
            __syncthreads();  // this stage has arrived, the one before has been read
            if (i + 1 < x.n1) fetch(half ^ 1);
            if (idle) return;
            const char *qt = lds + half * SB;
            f32x16_t s, u;
            kv_products<V, D>(qt, a.scale, s, u, w);
            kv_add_v<V, D>(qt, s, w);
            kv_add_k<V, D>(qt, u, w);
        };
        for (int i = x.n0; i < x.n1; i += 2) {
            step(i, 0);
            if (i + 1 < x.n1) step(i + 1, 1);
        }
    }
    const uint32_t odd = x.odd(a, w.dk[0][0]);
    x.template store<D>(a, 0, 0, w.dk, a.tau, odd);
    x.template store<D>(a, 1, 0, w.dv, 1.f, odd);
    if (odd) x.plain(a, odd);
}

// 32 rows of the states for all four waves, each on its own tiles of queries, staged for the
// wave alone: for problems too few to fill the CUs by 128 rows.  (d 32: the registers of float32
// held down for a third wave to a SIMD, 161 for 169: 46.1 for 47.7 microseconds at 4 x 8 heads of
// 700 x 900.)
template <typename S, int D>
__global__ __launch_bounds__(256, D == 128 ? 1 : D == 64 ? 2 : 3) void cross_dkdv_narrow_kernel(Gradients a, int items) {
    typedef Tile<S, D> X;
    constexpr int NB = kPrivate<S>, N = D / 32, SB = 2 * X::bytes(32) + 256;
    __shared__ __attribute__((aligned(16))) char lds[4 * NB * SB > 16384 * N ? 4 * NB * SB : 16384 * N];
    const int blk = blockIdx.y * gridDim.x + blockIdx.x;
    if (blk >= items) return;
    const int item = xcd_item(blk, items);
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tile = item % a.key_tiles, piece = item / a.key_tiles % a.dkv_pieces;
    const KvItem<S, D> x(a, item / a.key_tiles / a.dkv_pieces, 32 * tile, piece);
    typedef typename KvValue<S, D>::type V;
    KvRows<V, D> w;
#pragma unroll
    for (int dt = 0; dt < N; ++dt) w.dk[dt] = w.dv[dt] = zero16();
    if (32 * tile < x.len) {
        char *mine = lds + NB * SB * wv;
        int i = x.n0 + wv, buf = 0;
        auto at = x.tile_at(a, i);  // of the tile that is fetched
        if (i < x.n1) {
            x.template fetch_g<1>(a, at, mine, 0);
            x.template fetch_q<1>(a, at, mine, 0);
        }
        x.load(a, w);
        wait_loads<0>();  // k and v too: no wait for them stays in the loop
        for (; i < x.n1; i += 4, buf ^= NB - 1) {
            const bool more = i + 4 < x.n1;
            char *qt = mine + SB * buf, *next = mine + SB * (buf ^ (NB - 1));
            wait_loads<0>();
            wait_lds();
            x.step(a, at, 4);
            if (NB == 2 && more) {
                x.template fetch_g<1>(a, at, next, 0);
                x.template fetch_q<1>(a, at, next, 0);
            }
            f32x16_t s, u;
            kv_products<V, D>(qt, a.scale, s, u, w);
            kv_add_v<V, D>(qt, s, w);
            if (NB == 1 && more) {
                wait_lds();  // dO has been read
                x.template fetch_g<1>(a, at, qt, 0);
            }
            kv_add_k<V, D>(qt, u, w);
            if (NB == 1 && more) {
                wait_lds();  // q has been read
                x.template fetch_q<1>(a, at, qt, 0);
            }
        }
    }
    uint32_t odd = 0;  // as in dq
    add_waves<N>(w.dk, lds, wv, [&](int dt, const f32x16_t &sum) {
        odd = x.odd(a, sum[0]);
        x.template store<32>(a, 0, 32 * dt, &sum, a.tau, odd);
    });
    add_waves<N>(w.dv, lds, wv, [&](int dt, const f32x16_t &sum) { x.template store<32>(a, 1, 32 * dt, &sum, 1.f, odd); });
    odd &= every<N>(wv);
    if (odd) x.plain(a, odd);
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
    hipError_t e = launch(kCrossBwdDq, a.dq_narrow ? cross_dq_narrow_kernel<S, D> : cross_dq_kernel<S, D>, grid_of(n),
                          dim3(256), 0, st, a, (int)n);
    if (e != hipSuccess) return e;
    e = launch(kCrossBwdDkDv, a.dkv_narrow ? cross_dkdv_narrow_kernel<S, D> : cross_dkdv_kernel<S, D>, grid_of(m),
               dim3(256), 0, st, a, (int)m);
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

// Microseconds a wave needs for a tile of 32 x 32 while it has its SIMD alone, dq, or dk and
// dv: measured at 8 x 8 heads of 1024 x 1024, d 64, and 2 x 16 of 1000 x 2500, d 128, in
// bfloat16, and at 2 x 8 heads of 333 x 777, d 64, in float32.
double tile_us(int dtype, int D, bool dkv) {
    if (dtype == 1) return dkv ? 0.63 + 0.0112 * D : 0.75 + 0.003 * D;
    return (dkv ? (D == 128 ? 0.07 : 0.062) : 0.042) * D;
}

// How a gradient over `rows` rows to a problem is computed: narrow workgroups (32 rows, the
// other side's tiles divided among the waves) or wide ones (128 rows), and in how many pieces
// of the other side's n tiles: the least of an estimate of the time.  Wide and narrow dk,
// dv measured, in their best pieces, without the pieces' sum: 117 and 201 microseconds at 2 x 16
// heads on 4 of 1000 x 2500, d 128, bfloat16; 32 (two or more pieces) and 30 (one) at 4 x 8 heads
// of 200 x 200, d 128, float32.
void divide(int dtype, int D, long long prob, int rows, int n, bool dkv, int *narrow, int *tiles, int *pieces) {
    const double us = tile_us(dtype, D, dkv);
    double best = 1e30;
    for (int wide = 0; wide < 2; ++wide) {
        const int t = (rows + (wide ? 127 : 31)) / (wide ? 128 : 32);
        // float32 d 128 and the narrow kernel of bfloat16 d 128 leave no room for a second workgroup
        const double second = D == 128 && (dtype == 0 || !wide) ? 1.0 : 0.75;
        for (int p = 1; p <= 64 && p <= n; p += p < 4 ? 1 : p < 8 ? 2 : p < 16 ? 4 : 8) {
            const int each = wide ? (n + p - 1) / p : (n + 4 * p - 1) / (4 * p);
            const long long c = (prob * t * p + 255) / 256;  // workgroups to a CU
            if (p > 1 && c > 8) break;  // there are enough without more pieces
            double x = (each * us + 3.0) * (c == 1 ? 1.0 : c * second);
            if (p > 1) x += 3.0 + p * (dkv ? 2.0 : 1.0) * prob * rows * D * 8e-6 / 3.0;
            if (x < best) {
                best = x;
                *narrow = !wide;
                *tiles = t;
                *pieces = p;
            }
        }
    }
}

}  // namespace

void plan_cross_backward(int dtype, int D, Gradients *a) {
    const long long prob = (long long)a->Bkv * a->Hkv;
    divide(dtype, D, prob, a->rows, (a->S + 31) / 32, false, &a->dq_narrow, &a->row_tiles, &a->dq_pieces);
    // a tile of queries is of one head and one batch entry, however few positions it has
    divide(dtype, D, prob, a->S, (a->T + 31) / 32 * a->G * a->share, true, &a->dkv_narrow, &a->key_tiles,
           &a->dkv_pieces);
}

hipError_t launch_cross_backward(int dtype, int D, const Gradients &a, hipStream_t s) {
    return dtype == 1 ? backward_d<uint16_t>(D, a, s) : backward_d<float>(D, a, s);
}

}  // namespace fibattn
