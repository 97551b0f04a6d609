// Dense attention of queries to states of another length, and the join of partial results.
//
//   s_rj = tau <q_r, k_j>,  o_r = sum_j exp(s_rj - lse_r) v_j,  lse_r = log sum_j exp(s_rj)
// in one pass over j with the running maximum and sum of each row, in float32.
#include "cross_launch.h"

namespace fibattn {

namespace {

// A workgroup of 8 waves on 32 RW query rows: RW waves side by side, KW = 8 / RW waves to the
// same rows, each on its own 32 of the staged rows of the states.  Two waves to the same rows
// double the waves a CU holds (MFMA and exponentials of one wave run beside another's)
// without a result in memory.
template <typename S, int D, int RW> struct Shape {
    static constexpr int KW = 8 / RW;
    static constexpr int NT = 32 * KW;                   // rows of a stage
    static constexpr int TB = Tile<S, D>::bytes(NT);     // bytes of its k, and of its v
    static constexpr int merge = RW * (KW - 1) * 32 * (D + 2) * 4;
    static constexpr int lds = 4 * TB > merge ? 4 * TB : merge;
};

template <typename S, int D> constexpr int keys_lds() {
    // per wave: K and V of 32 rows; at the end the waves' results
    constexpr int waves = 4 * 2 * Tile<S, D>::bytes(32), merge = 4 * 32 * D * 4;
    return waves > merge ? waves : merge;
}

// A wave's 32 query rows.
template <typename S, int D> struct Rows {
    Frag<S> q[D / 16];
    f32x16_t acc[D / 32];  // transposed: column = row of the lane
    float m, l;            // running maximum (in powers of two) and the lane's own part of the sum
    float neg, top;        // -m, or 0 while m is -inf; the logit above which m moves
    int lim;               // rows of the states that this row reads
    long long id;          // (b H + h) T + t
    RowAt at;
    bool on;
};

template <typename S, int D>
__device__ __forceinline__ void load_rows(const Queries &a, const States &st, int b0, int j, int r0, int len,
                                          Rows<S, D> &w) {
    const int lane = threadIdx.x & 63, h = lane >> 5, r = r0 + (lane & 31);
    w.on = r < st.rows;
    w.at = row_at(a, b0, j, min(r, st.rows - 1));
    w.id = ((long long)w.at.b * a.H + w.at.h) * a.T + w.at.t;
    w.lim = st.causal ? min(len - a.T + 1 + w.at.t, len) : len;
    const S *row = (const S *)a.q + w.at.b * a.lq.sb + w.at.h * a.lq.sh + w.at.t * a.lq.st;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) load_frag(row, ks, h, w.q[ks]);
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) w.acc[dt] = zero16();
    w.m = w.top = -INFINITY;
    w.l = w.neg = 0.f;
}

template <typename S, int D>
__device__ __forceinline__ f32x16_t logits(const char *kt, int row0, const Rows<S, D> &w) {
    const int lane = threadIdx.x & 63;
    f32x16_t s = zero16();
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
        Frag<S> f;
        Tile<S, D>::row_frag(kt, row0 + (lane & 31), ks, lane >> 5, f);
        s = mma(f, w.q[ks], s);
    }
    return s;
}

// Rows of the states from `base` that a query does not read count nothing.
template <typename S, int D>
__device__ __forceinline__ void mask(f32x16_t &s, int base, const Rows<S, D> &w) {
    const int h = (threadIdx.x >> 5) & 1;
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (base + 8 * (i >> 2) + 4 * h + (i & 3) >= w.lim) s[i] = -INFINITY;
}

// A reference m from here on is rounded by up to 16 powers of two and more: a weight
// exp2(s scale - m), whose product is not rounded, may be 0 for the largest logit too, and the
// row is done again (again()).
__device__ __forceinline__ bool coarse(float m) { return fabsf(m) >= 0x1p28f && fabsf(m) < INFINITY; }

// Logits to weights exp2(s - m).  The reference m moves only when a logit passes it by 8
// powers of two: the sums keep their 24 bits and the accumulators are rarely rescaled.  What a
// tile has to look at is the lane's own maximum; the halves' common one is taken with the move.
// A coarse m is a step up, so that no weight passes 1, and moves with every tile: sums that
// are not used in the end (a larger m follows, or the row is done again) stay finite.
template <typename S, int D>
__device__ __forceinline__ void weights(f32x16_t &s, float scale, Rows<S, D> &w) {
    float top = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
    if (__ballot(top > w.top)) {
        float m = half_max(top) * scale;
        if (coarse(m)) m = fmaf(fabsf(m), 0x1p-23f, m);
        m = fmaxf(m, w.m);
        const float f = m == -INFINITY ? 1.f : ex2(w.m - m);
        w.m = m;
        w.neg = m == -INFINITY ? 0.f : -m;
        w.top = coarse(m) ? -INFINITY : (m + 8.f) * __builtin_amdgcn_rcpf(scale);
        w.l *= f;
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) w.acc[dt] *= f;
    }
    float l = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        s[i] = ex2(fmaf(s[i], scale, w.neg));
        l += s[i];
    }
    w.l += l;
}

template <typename S, int D>
__device__ __forceinline__ void values(const char *vt, int row0, const f32x16_t &p, Rows<S, D> &w) {
#pragma unroll
    for (int a = 0; a < 2; ++a) {
        const Weights<S> pw(p, a);
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) {
            Frag<S> f;
            Tile<S, D>::operand_t(vt, row0 + 16 * a, dt, f);
            w.acc[dt] = pw.add(f, w.acc[dt]);
        }
    }
}

// o and lse of a row (or its partial results), from the sum l over both halves.
__device__ __forceinline__ void store_lse(const Queries &a, long long slot, long long id, float z) {
    if (a.part_lse)
        a.part_lse[slot * a.B * a.H * a.T + id] = z;
    else
        a.lse[id] = z;
}
__device__ __forceinline__ void put_lse(const Queries &a, long long slot, long long id, float m, float l) {
    store_lse(a, slot, id, l == 0.f ? -INFINITY : (m + __log2f(l)) * kLn2);
}

template <typename S, int D>
__device__ __forceinline__ S *out_row(const Queries &a, const RowAt &at) {
    return (S *)a.o + at.b * a.lo.sb + at.h * a.lo.sh + at.t * a.lo.st;
}

// Rows of a tile that are to be done again (bit i: row r0 + i), over rows [c0, c1) of the states.
struct Redo {
    uint32_t which;
    int b0, j, r0, c0, c1, len;
    long long slot;
};
// Whether a row's sum is one that the tiles may have made not finite: of the weights l, some of
// its values' sums are not.  (A bfloat16 row whose weights are NaN met a NaN among what it reads;
// a float32 one may have met an infinity, of which the parts of a value make a NaN.)  Or one
// whose reference m is coarse, so that its weights may all be 0.
template <typename S> __device__ __forceinline__ bool again(float values, float l, float m) {
    return coarse(m) || (!(fabsf(values) < INFINITY) && (sizeof(S) == 4 || l == l));
}

// 32 RW query rows, 32 to a wave; the waves share the staged rows of the states.
template <typename S, int D, int RW>
__device__ __forceinline__ void rows_body(const Queries &a, const States &st, int item, char *lds, Redo &todo) {
    typedef Tile<S, D> X;
    typedef Shape<S, D, RW> Y;
    constexpr int NT = Y::NT, KW = Y::KW, TB = Y::TB;
    const int lane = threadIdx.x & 63, h = lane >> 5, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rw = wv % RW, kw = wv / RW;
    const int tile = item % st.tiles, piece = item / st.tiles % st.splits, prob = item / st.tiles / st.splits;
    const int b0 = prob / a.Hkv, j = prob % a.Hkv, r0 = 32 * (RW * tile + rw);
    const int len = states_len(st, b0);
    Rows<S, D> w;
    load_rows<S, D>(a, st, b0, j, r0, len, w);
    const bool idle = r0 >= st.rows;

    const int n = (len + NT - 1) / NT;
    const int n0 = (int)((long long)n * piece / st.splits), n1 = (int)((long long)n * (piece + 1) / st.splits);
    const int low = st.causal ? max(len - a.T + 1, 0) : len;  // rows that every query reads
    const char *kp = (const char *)((const S *)st.k + b0 * st.lk.sb + j * st.lk.sh);
    const char *vp = (const char *)((const S *)st.v + b0 * st.lv.sb + j * st.lv.sh);
    const long long ks = st.lk.st * (long long)sizeof(S), vs = st.lv.st * (long long)sizeof(S);
    auto fetch = [&](int i, int half) {
        const int r = i * NT;
        char *dst = lds + half * 2 * TB;
        X::template stage<NT, 8>(dst, kp + r * ks, ks, len - r, wv);
        X::template stage<NT, 8>(dst + TB, vp + r * vs, vs, len - r, wv);
    };
    if (n0 < n1) fetch(n0, 0);
    wait_loads<0>();  // the queries too: no wait for them stays in the loop
    // one stage from half `half` of the LDS; two to a turn of the loop, so that their addresses
    // are constants (-3 % at 2048 x 8192, d 64)
    auto step = [&](int i, int half) {
        wait_loads<0>();
        __syncthreads();  // this stage has arrived, the one before has been read
        if (i + 1 < n1) fetch(i + 1, half ^ 1);
        const int base = i * NT + 32 * kw;
        if (idle || base >= len) return;
        const char *kt = lds + half * 2 * TB, *vt = kt + TB;
        f32x16_t s = logits<S, D>(kt, 32 * kw, w);
        if (base + 32 > low) mask<S, D>(s, base, w);
        weights<S, D>(s, a.scale, w);
        values<S, D>(vt, 32 * kw, s, w);
    };
    for (int i = n0; i < n1; i += 2) {
        step(i, 0);
        if (i + 1 < n1) step(i + 1, 1);
    }
    float l = half_sum(w.l);
    if (KW > 1) {
        // the waves of the same rows, joined in their order; lanes hold the same places
        __syncthreads();
        float *part = (float *)lds + (rw * (KW - 1)) * 32 * (D + 2);
        if (kw) {
            float *x = part + (kw - 1) * 32 * (D + 2);
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                for (int e = 0; e < 16; e += 4)
                    *reinterpret_cast<f32x4_t *>(x + (dt * 16 + e) * 64 + 4 * lane) =
                        f32x4_t{w.acc[dt][e], w.acc[dt][e + 1], w.acc[dt][e + 2], w.acc[dt][e + 3]};
            x[32 * D + lane] = h ? l : w.m;
        }
        __syncthreads();
        if (kw) return;
#pragma unroll 1
        for (int o = 0; o < KW - 1; ++o) {
            const float *x = part + o * 32 * (D + 2);
            const float m2 = x[32 * D + (lane & 31)], l2 = x[32 * D + 32 + (lane & 31)], m = fmaxf(w.m, m2);
            // a wave that met no rows has the maximum -inf: it counts nothing
            const float f1 = w.m == -INFINITY ? 0.f : ex2(w.m - m), f2 = m2 == -INFINITY ? 0.f : ex2(m2 - m);
            w.m = m;
            l = l * f1 + l2 * f2;
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                for (int e = 0; e < 16; e += 4) {
                    const f32x4_t y = *reinterpret_cast<const f32x4_t *>(x + (dt * 16 + e) * 64 + 4 * lane);
#pragma unroll
                    for (int z = 0; z < 4; ++z) w.acc[dt][e + z] = w.acc[dt][e + z] * f1 + y[z] * f2;
                }
        }
    }
    const float f = l == 0.f ? 0.f : 1.f / l;
    const long long slot = st.slot + piece;
    float odd = 0.f;  // NaN if a value is not finite
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) odd = fmaf(w.acc[dt][e], 0.f, odd);
    const unsigned long long bad = __ballot(w.on && again<S>(odd, l, w.m));
    if (bad) todo = {(uint32_t)(bad | bad >> 32), b0, j, r0, n0 * NT, min(n1 * NT, len), len, slot};
    if (!w.on || (todo.which >> (lane & 31) & 1)) return;
    if (h == 0) put_lse(a, slot, w.id, w.m, l);
    if (a.part_o)
        store_cols<D>(a.part_o + (slot * a.B * a.H * a.T + w.id) * D, w.acc, f, h);
    else
        store_cols<D>(out_row<S, D>(a, w.at), w.acc, f, h);
}

// 32 query rows for all four waves, each on its own rows of the states (tiles of 32, one in
// four), staged for the wave alone; joined in LDS.
template <typename S, int D>
__device__ __forceinline__ void keys_body(const Queries &a, const States &st, int item, char *lds, Redo &todo) {
    typedef Tile<S, D> X;
    constexpr int TB = X::bytes(32), OPS = 32 / X::kRowsPerLoad;
    __shared__ float stat[2][4][32];
    __shared__ uint32_t odd_rows[32];
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    const int tile = item % st.tiles, piece = item / st.tiles % st.splits, prob = item / st.tiles / st.splits;
    const int b0 = prob / a.Hkv, j = prob % a.Hkv;
    const int len = states_len(st, b0);
    Rows<S, D> w;
    load_rows<S, D>(a, st, b0, j, 32 * tile, len, w);
    const int n = (len + 31) / 32;
    const int n0 = (int)((long long)n * piece / st.splits), n1 = (int)((long long)n * (piece + 1) / st.splits);
    const int low = st.causal ? max(len - a.T + 1, 0) : len;
    const char *kp = (const char *)((const S *)st.k + b0 * st.lk.sb + j * st.lk.sh);
    const char *vp = (const char *)((const S *)st.v + b0 * st.lv.sb + j * st.lv.sh);
    const long long ks = st.lk.st * (long long)sizeof(S), vs = st.lv.st * (long long)sizeof(S);
    char *kt = lds + 2 * TB * wv, *vt = kt + TB;
    int i = n0 + wv;
    if (i < n1) {
        X::template stage<32, 1>(kt, kp + 32 * i * ks, ks, len - 32 * i, 0);
        X::template stage<32, 1>(vt, vp + 32 * i * vs, vs, len - 32 * i, 0);
    }
    for (; i < n1; i += 4) {
        const bool more = i + 4 < n1;
        wait_loads<OPS>();  // K is here, V may be on its way
        f32x16_t s = logits<S, D>(kt, 0, w);
        wait_lds();  // K has been read
        if (more) X::template stage<32, 1>(kt, kp + 32 * (i + 4) * ks, ks, len - 32 * (i + 4), 0);
        if (32 * (i + 1) > low) mask<S, D>(s, 32 * i, w);
        weights<S, D>(s, a.scale, w);
        if (more)
            wait_loads<OPS>();
        else
            wait_loads<0>();
        values<S, D>(vt, 0, s, w);
        wait_lds();  // V has been read
        if (more) X::template stage<32, 1>(vt, vp + 32 * (i + 4) * vs, vs, len - 32 * (i + 4), 0);
    }
    // the waves' results of each row, in the order of the waves
    const float l = half_sum(w.l);
    __syncthreads();
    float *part = (float *)lds;
    store_cols<D>(part + (32 * wv + (lane & 31)) * D, w.acc, 1.f, h);
    if (h == 0) {
        stat[0][wv][lane] = w.m;
        stat[1][wv][lane] = l;
    }
    if (threadIdx.x < 32) odd_rows[threadIdx.x] = 0;
    __syncthreads();
    constexpr int V = 4, per = D / V, each = 32 * per / 256;  // lanes to a row, values of a lane
    f32x4_t y[each];
    float lse[each];
#pragma unroll
    for (int e = 0; e < each; ++e) {
        const int r = (threadIdx.x + 256 * e) / per, d = (threadIdx.x + 256 * e) % per * V;
        float m = stat[0][0][r];
#pragma unroll
        for (int x = 1; x < 4; ++x) m = fmaxf(m, stat[0][x][r]);
        float sum = 0.f;
        y[e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            // a wave that met no rows has the maximum -inf: it counts nothing
            const float f = stat[0][x][r] == -INFINITY ? 0.f : ex2(stat[0][x][r] - m);
            sum += stat[1][x][r] * f;
            y[e] += *reinterpret_cast<const f32x4_t *>(part + (32 * x + r) * D + d) * f;
        }
        if (again<S>((y[e][0] + y[e][1]) * 0.f + (y[e][2] + y[e][3]) * 0.f, sum, m)) odd_rows[r] = 1;
        y[e] *= sum == 0.f ? 0.f : 1.f / sum;
        lse[e] = sum == 0.f ? -INFINITY : (m + __log2f(sum)) * kLn2;
    }
    __syncthreads();
    const long long slot = st.slot + piece;
    const uint32_t odd = (uint32_t)__ballot(odd_rows[lane & 31] != 0);
#pragma unroll
    for (int e = 0; e < each; ++e) {
        const int r = (threadIdx.x + 256 * e) / per, d = (threadIdx.x + 256 * e) % per * V;
        if (32 * tile + r >= st.rows || (odd >> r & 1)) continue;
        const RowAt at = row_at(a, b0, j, 32 * tile + r);
        const long long id = ((long long)at.b * a.H + at.h) * a.T + at.t;
        if (d == 0) store_lse(a, slot, id, lse[e]);
        if (a.part_o) {
            *reinterpret_cast<f32x4_t *>(a.part_o + (slot * a.B * a.H * a.T + id) * D + d) = y[e];
        } else {
            S *row = out_row<S, D>(a, at) + d;
            if constexpr (sizeof(S) == 4)
                *reinterpret_cast<f32x4_t *>(row) = y[e];
            else
                *reinterpret_cast<uint2 *>(row) = make_uint2(pack2(y[e][0], y[e][1]), pack2(y[e][2], y[e][3]));
        }
    }
    // of the rows this problem has, a wave to every fourth
    const int rows = st.rows - 32 * tile;
    const uint32_t which = odd & (0x11111111u << wv) & (rows < 32 ? (1u << rows) - 1 : ~0u);
    if (which) todo = {which, b0, j, 32 * tile, 32 * n0, min(32 * n1, len), len, slot};
}

// x y, rounded whatever is done with it next.
__device__ __forceinline__ float rounded(float x, float y) {
#pragma clang fp contract(off)
    return x * y;
}

// The rows of `todo`, each by the whole wave: a lane to each of 64 rows of the states, and only
// to those that the query reads, for the weights; a lane to each value for the sums.
//
// The tiles multiply what a query does not read by a weight of 0, and the rest of a weight may
// be 0 or negative: with an infinity or NaN among the values either makes a NaN of what is not
// one.  Here nothing unread enters, every weight is whole, and a logit is rounded before the
// largest one is subtracted from it, whose weight then is 1.  There are at most 2^30 weights of at
// most 1: 2^-31 of them, and the 2^31 with the division by their sum, keep the sums of large values
// from overflowing as the tiles' may (bits are lost of products below 2^-94).
template <typename S, int D>
__device__ __forceinline__ void plain_rows(const Queries &a, const States &st, const Redo &todo) {
    constexpr int N = (D + 63) / 64;
    const int lane = threadIdx.x & 63;
    const S *k = (const S *)st.k + todo.b0 * st.lk.sb + todo.j * st.lk.sh;
    const S *v = (const S *)st.v + todo.b0 * st.lv.sb + todo.j * st.lv.sh;
    for (uint32_t left = todo.which; left; left &= left - 1) {
        const RowAt at = row_at(a, todo.b0, todo.j, todo.r0 + __builtin_ctz(left));
        const long long id = ((long long)at.b * a.H + at.h) * a.T + at.t;
        const S *q = (const S *)a.q + at.b * a.lq.sb + at.h * a.lq.sh + at.t * a.lq.st;
        const int lim = min(st.causal ? todo.len - a.T + 1 + at.t : todo.len, todo.c1);
        float y[N], m = -INFINITY, l = 0.f;
#pragma unroll
        for (int n = 0; n < N; ++n) y[n] = 0.f;
        for (int c = todo.c0; c < lim; c += 64) {
            float s = -INFINITY;
            if (c + lane < lim) s = rounded(dot_row<S, D>(q, k + (c + lane) * st.lk.st), a.scale);
            // a NaN stays one: fmaxf drops it, its weight below does not
            float top = s;
#pragma unroll
            for (int e = 32; e; e >>= 1) top = fmaxf(top, __shfl_xor(top, e, 64));
            top = fmaxf(top, m);
            const float f = top == -INFINITY ? 1.f : ex2(m - top);
            const float p = c + lane < lim ? ex2(s - (top == -INFINITY ? 0.f : top)) : 0.f;
            float sum = p;
#pragma unroll
            for (int e = 32; e; e >>= 1) sum += __shfl_xor(sum, e, 64);
            m = top;
            l = fmaf(l, f, sum);
#pragma unroll
            for (int n = 0; n < N; ++n) y[n] *= f;
            const int count = min(64, lim - c);
            for (int e = 0; e < count; ++e) {
                const float w = __shfl(p, e, 64) * 0x1p-31f;
#pragma unroll
                for (int n = 0; n < N; ++n)
                    if (lane + 64 * n < D) y[n] = fmaf(w, value_of(v[(c + e) * st.lv.st + lane + 64 * n]), y[n]);
            }
        }
        const float f = l == 0.f ? 0.f : 0x1p31f / l;
        if (lane == 0) put_lse(a, todo.slot, id, m, l);
#pragma unroll
        for (int n = 0; n < N; ++n)
            if (lane + 64 * n < D) {
                if (a.part_o)
                    a.part_o[(todo.slot * a.B * a.H * a.T + id) * D + lane + 64 * n] = y[n] * f;
                else
                    put_value(out_row<S, D>(a, at) + lane + 64 * n, y[n] * f);
            }
    }
}

// By rows (RW > 0: 8 waves) or by keys (RW 0: 4 waves).
template <typename S, int D, int RW>
__device__ __forceinline__ void body(const Queries &a, const States &st, int item, char *lds) {
    Redo todo;
    todo.which = 0;
    if constexpr (RW == 0)
        keys_body<S, D>(a, st, item, lds, todo);
    else
        rows_body<S, D, RW>(a, st, item, lds, todo);
    if (todo.which) plain_rows<S, D>(a, st, todo);
}

template <typename S, int D, int RW> constexpr int body_lds() {
    if constexpr (RW == 0)
        return keys_lds<S, D>();
    else
        return Shape<S, D, RW>::lds;
}

// Waves to a SIMD that the registers are held down for.
template <typename S, int D, int RW> constexpr int simd_waves() {
    if (sizeof(S) == 4 && D == 128) return RW ? 2 : 1;
    return D * (int)sizeof(S) <= 128 && RW ? 4 : 2;
}

// Items [0, n0) of s0, then those of s1.
template <typename S, int D, int RW>
__global__ __launch_bounds__(RW ? 512 : 256, (simd_waves<S, D, RW>())) void cross_fwd_kernel(Queries a, States s0,
                                                                                          States s1, int n0, int n) {
    __shared__ __attribute__((aligned(16))) char lds[body_lds<S, D, RW>()];
    const int b = blockIdx.y * gridDim.x + blockIdx.x;
    if (b >= n) return;
    const bool first = b < n0;
    body<S, D, RW>(a, first ? s0 : s1, first ? xcd_item(b, n0) : xcd_item(b - n0, n - n0), lds);
}

// Partial results of a row: o = sum_i exp(lse_i - lse) o_i, lse = log sum_i exp(lse_i).  A
// part without rows (lse -inf) counts nothing, whatever its o holds.  A wave to a row: lane i
// has the weights of parts i and 64 + i (there are at most 128), of sum 1, so that no sum of
// values overflows; D / 4 lanes add every (256 / D)-th part.
template <typename S, int D>
__global__ __launch_bounds__(256) void join_parts_kernel(Queries a, int parts) {
    constexpr int per = D / 4, groups = 64 / per;
    const long long rows = (long long)a.B * a.H * a.T;
    const long long r = ((long long)blockIdx.y * gridDim.x + blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (r >= rows) return;
    const int lane = threadIdx.x & 63, g = lane / per, d = lane % per * 4;
    float z[2], f[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) z[c] = lane + 64 * c < parts ? a.part_lse[(lane + 64 * c) * rows + r] : -INFINITY;
    float m = fmaxf(z[0], z[1]);
#pragma unroll
    for (int e = 32; e; e >>= 1) m = fmaxf(m, __shfl_xor(m, e, 64));
#pragma unroll
    for (int c = 0; c < 2; ++c) f[c] = z[c] == -INFINITY ? 0.f : ex2((z[c] - m) * kLog2e);
    float sum = f[0] + f[1];
#pragma unroll
    for (int e = 32; e; e >>= 1) sum += __shfl_xor(sum, e, 64);
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    f32x4_t y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const int n = min(64, parts - 64 * c);
        f[c] *= inv;
        const float *x = a.part_o + ((long long)(64 * c) * rows + r) * D + d;
        for (int first = 0; first < n; first += 4 * groups) {
            f32x4_t v[4];  // four parts on their way at a time
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int i = first + u * groups + g;
                v[u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
                if (i < n) v[u] = *reinterpret_cast<const f32x4_t *>(x + (long long)i * rows * D);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float w = __shfl(f[c], min(first + u * groups + g, 63), 64);
                if (first + u * groups + g < n && w != 0.f) y += v[u] * w;
            }
        }
    }
#pragma unroll
    for (int e = 32; e >= per; e >>= 1)
#pragma unroll
        for (int c = 0; c < 4; ++c) y[c] += __shfl_xor(y[c], e, 64);
    if (g) return;
    const int t = (int)(r % a.T), h = (int)(r / a.T % a.H), b = (int)(r / a.T / a.H);
    if (d == 0) a.lse[r] = sum == 0.f ? -INFINITY : m + __log2f(sum) * kLn2;
    S *row = out_row<S, D>(a, {b, h, t}) + d;
    if constexpr (sizeof(S) == 4)
        *reinterpret_cast<f32x4_t *>(row) = y;
    else
        *reinterpret_cast<uint2 *>(row) = make_uint2(pack2(y[0], y[1]), pack2(y[2], y[3]));
}

// The same for two stored results over disjoint sets of keys, whose rounding to the storage type
// (2^-8 of each in bfloat16) they bring with them; partial results of one call are float32.
template <typename S, int D>
__global__ __launch_bounds__(256) void join_kernel(JoinArgs a) {
    constexpr int N = 16 / (int)sizeof(S), per = D / N;
    const long long rows = (long long)a.B * a.H * a.T;
    const long long e = ((long long)blockIdx.y * gridDim.x + blockIdx.x) * 256 + threadIdx.x;
    const long long r = e / per;
    const int d = (int)(e % per) * N;
    if (r >= rows) return;
    const int t = (int)(r % a.T), h = (int)(r / a.T % a.H), b = (int)(r / a.T / a.H);
    const float za = a.za[r], zb = a.zb[r];
    const float m = fmaxf(za, zb);
    const float fa = za == -INFINITY ? 0.f : ex2((za - m) * kLog2e), fb = zb == -INFINITY ? 0.f : ex2((zb - m) * kLog2e);
    const float sum = fa + fb, f = sum == 0.f ? 0.f : 1.f / sum;
    float x[N], y[N], o[N];
    Vec<S>::load((const S *)a.a + b * a.la.sb + h * a.la.sh + t * a.la.st + d, x);
    Vec<S>::load((const S *)a.b + b * a.lb.sb + h * a.lb.sh + t * a.lb.st + d, y);
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = (fa == 0.f ? 0.f : x[i] * fa * f) + (fb == 0.f ? 0.f : y[i] * fb * f);
    Vec<S>::store((S *)a.o + b * a.lo.sb + h * a.lo.sh + t * a.lo.st + d, o);
    if (d == 0) a.z[r] = sum == 0.f ? -INFINITY : m + __log2f(sum) * kLn2;
}

// By rows or by keys, row tiles and pieces of states for `prob` problems: the least of an
// estimate of the time.  A wave takes 0.007 D microseconds for a tile of 32 x 32 in bfloat16,
// 0.022 D in float32; two waves to a SIMD take 1.5 times as long as one.  By rows and by keys
// measured, each in its best pieces: 35 and 51 microseconds at 8 x 8 heads of 1024 x 1024, d 64,
// bfloat16; 41 and 28 (both launches and the join) where 64 sequences of 16 heads on 4 share 8192
// rows, d 128.  joined: the call has a join in any case; else pieces add its launch, 5 microseconds.
// (Against 3 in both cases, of drawn shapes for which it matters: 1.04 times as fast in a graph
// and 1.09 from the host in 40 without, 1.02 and 1.00 in 30 with other states.)  beside: how
// states of the same call are read, whose launch these share if they are read so too (-1: none).
void plan(int dtype, int D, States *s, int prob, bool joined, int beside = -1) {
    const double us = (dtype == 1 ? 0.007 : 0.022) * D, row = 2.0 * D * (dtype == 1 ? 2 : 4);
    const int n = (s->S + 31) / 32;
    double best = 1e30;
    for (int rw = 0; rw <= 4; rw += 4) {
        const int per = rw ? 128 : 32, t = (s->rows + per - 1) / per;
        // the states' rows, read once from memory and by every row tile from L2
        const double once = (double)prob * s->S * row / 5e6, all = once * t * (5e6 / 1.2e7);
        for (int p = 1; p <= 64 && p <= n; p += p < 4 ? 1 : p < 8 ? 2 : p < 16 ? 4 : 8) {
            const long long c = ((long long)prob * t * p + 255) / 256;  // workgroups to a CU
            if (p > 1 && c > 8) break;  // there are enough without more pieces
            const double each = rw ? 1.5 * us * ((n + 2 * p - 1) / (2 * p)) : us * ((n + 4 * p - 1) / (4 * p));
            // float32 rows of 128 leave no room for a second workgroup
            double x = (each + 3.0) * (c == 1 ? 1.0 : c * (dtype == 0 && D == 128 ? 1.0 : 0.75));
            const double busy = c > 1 ? 1.0 : (double)prob * t * p / 256;
            const double read = (once > all ? once : all) / busy + 3.0;
            if (read > x) x = read;
            if (beside >= 0 && rw != beside) x += 4.0;
            if (p > 1) x += (joined ? 1.5 : 5.0) + p * (double)prob * s->rows * D * 8e-6 / 3.0;
            if (x < best) {
                best = x;
                s->rw = rw;
                s->tiles = t;
                s->splits = p;
            }
        }
    }
}

template <typename S, int D, int RW>
hipError_t launch_as(const Queries &q, const States &s0, const States &s1, long long n0, long long n, hipStream_t st) {
    if (n >= 1ll << 31) return hipErrorInvalidValue;
    return launch(kCrossForward, cross_fwd_kernel<S, D, RW>, grid_of(n, RW ? 512 : 256), dim3(RW ? 512 : 256), 0, st, q,
                  s0, s1, (int)n0, (int)n);
}
template <typename S, int D>
hipError_t launch_parts(const Queries &q, const States &s0, const States &s1, long long n0, long long n, hipStream_t st) {
    return s0.rw ? launch_as<S, D, 4>(q, s0, s1, n0, n, st) : launch_as<S, D, 0>(q, s0, s1, n0, n, st);
}

template <typename S, int D>
hipError_t forward(const Queries &a, const States &s0, const States *s1, int prob0, int prob1, hipStream_t st) {
    const int parts = s0.splits + (s1 ? s1->splits : 0);
    const long long n0 = (long long)prob0 * s0.tiles * s0.splits;
    const long long n1 = s1 ? (long long)prob1 * s1->tiles * s1->splits : 0;
    const States &own = s1 ? *s1 : s0;
    Queries q = a;
    if (parts == 1) q.part_o = q.part_lse = nullptr;
    // states that are read the same way share a launch
    const bool both = !s1 || own.rw == s0.rw;
    hipError_t e = launch_parts<S, D>(q, s0, own, n0, both ? n0 + n1 : n0, st);
    if (e == hipSuccess && !both) e = launch_parts<S, D>(q, own, own, n1, n1, st);
    if (e != hipSuccess || parts == 1) return e;
    const long long rows = (long long)a.B * a.H * a.T;
    return launch(kJoin, join_parts_kernel<S, D>, grid_of((rows + 3) / 4), dim3(256), 0, st, q, parts);
}

template <typename S>
hipError_t forward_d(int D, const Queries &a, const States &s0, const States *s1, int prob0, int prob1, hipStream_t st) {
    switch (D) {
        case 32: return forward<S, 32>(a, s0, s1, prob0, prob1, st);
        case 64: return forward<S, 64>(a, s0, s1, prob0, prob1, st);
        default: return forward<S, 128>(a, s0, s1, prob0, prob1, st);
    }
}

template <typename S> hipError_t join_d(int D, const JoinArgs &a, hipStream_t st) {
    const long long rows = (long long)a.B * a.H * a.T, per = D * (long long)sizeof(S) / 16;
    const dim3 grid = grid_of((rows * per + 255) / 256);
    switch (D) {
        case 32: return launch(kJoin, join_kernel<S, 32>, grid, dim3(256), 0, st, a);
        case 64: return launch(kJoin, join_kernel<S, 64>, grid, dim3(256), 0, st, a);
        default: return launch(kJoin, join_kernel<S, 128>, grid, dim3(256), 0, st, a);
    }
}

}  // namespace

int plan_cross_forward(int dtype, int D, States *s0, States *s1, int prob0, int prob1) {
    if (s1) plan(dtype, D, s1, prob1, true);
    plan(dtype, D, s0, prob0, s1 != nullptr, s1 ? s1->rw : -1);
    s0->slot = 0;
    if (!s1) return s0->splits;
    s1->slot = s0->splits;
    return s0->splits + s1->splits;
}

hipError_t launch_cross_forward(int dtype, int D, const Queries &a, const States &s0, const States *s1, int prob0,
                                int prob1, hipStream_t s) {
    return dtype == 1 ? forward_d<uint16_t>(D, a, s0, s1, prob0, prob1, s)
                      : forward_d<float>(D, a, s0, s1, prob0, prob1, s);
}

hipError_t launch_join(int dtype, int D, const JoinArgs &a, hipStream_t s) {
    return dtype == 1 ? join_d<uint16_t>(D, a, s) : join_d<float>(D, a, s);
}

}  // namespace fibattn
