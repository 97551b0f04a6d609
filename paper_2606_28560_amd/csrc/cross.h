// Dense attention to states that are not the sequence's own (an encoder's, a memory or a
// prefix that the batch shares): the pieces its kernels share.
//
// Every product runs on 32 x 32 matrix-core tiles.  A tile's operands hold, per lane, 8
// values of one row: lane l serves row l % 32 and the inner indices 8h .. 8h + 7 of a step
// of 16, h = l / 32 (Frag), one v_mfma_f32_32x32x16_bf16 a step.  The result holds column
// l % 32 and rows 8 (i / 4) + 4h + i % 4, i < 16.
//
// A float32 value goes as the sum of three bfloat16 ones, a = a0 + a1 + a2, each the rounded
// rest of those before: |a1| <= 2^-8 |a|, |a2| <= 2^-16 |a|, and no rest stays (24 bits in
// three times 8).  Of a product's nine partial products the six down to 2^-16 are taken, each
// exact, summed in float32; the two largest of the others are at most 2^-24 of it.  Six
// bfloat16 steps take 192 cycles of a matrix core where v_mfma_f32_32x32x2_f32 takes 512
// (with the parts' making, forward and dq 1.2 to 1.35 times as fast, dk and dv 1.1 to 1.2 at
// d 64 and 32).  The parts of d 128's rows of k and v are too many registers beside dk and dv:
// those kernels take the float32 instructions (whole_t; 29 against 40 microseconds at 4 x 8
// heads of 200 x 200).
//
// The kernels form the transposed logits, so that a lane holds one query's (dk, dv: one
// key's) weights: of 16 consecutive inner rows its half h has rows 4h .. 4h + 3 and
// 8 + 4h .. 8 + 4h + 3.  That is the operand of the next product when the other operand
// takes its inner rows in the same order (operand_t): no weight leaves its lane.
#pragma once

#include "common.h"

namespace fibattn {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef short i16x4_t __attribute__((ext_vector_type(4)));
typedef unsigned u32x4_t __attribute__((ext_vector_type(4)));

template <typename S> struct FragOf;
template <> struct FragOf<uint16_t> { typedef bf16x8_t type; };
struct bf16x8x3_t {
    bf16x8_t p[3];
};
template <> struct FragOf<float> { typedef bf16x8x3_t type; };
// float32 values that are multiplied whole: slot s of a step pairs inner indices s and 8 + s.
struct whole_t {
    float x;
};
template <> struct FragOf<whole_t> { typedef f32x8_t type; };
template <typename S> using Frag = typename FragOf<S>::type;

__device__ __forceinline__ f32x16_t mma(const bf16x8_t &a, const bf16x8_t &b, const f32x16_t &c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16_t mma(const bf16x8x3_t &a, const bf16x8x3_t &b, f32x16_t c) {
    c = mma(a.p[2], b.p[0], c);  // the small ones first
    c = mma(a.p[0], b.p[2], c);
    c = mma(a.p[1], b.p[1], c);
    c = mma(a.p[1], b.p[0], c);
    c = mma(a.p[0], b.p[1], c);
    return mma(a.p[0], b.p[0], c);
}

__device__ __forceinline__ f32x16_t mma(const f32x8_t &a, const f32x8_t &b, f32x16_t c) {
#pragma unroll
    for (int s = 0; s < 8; ++s) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[s], b[s], c, 0, 0, 0);
    return c;
}

__device__ __forceinline__ f32x16_t zero16() {
    return f32x16_t{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
}

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    const f32x2_t v = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2_t));
}

// x in N bfloat16 parts.  (The rest of a rounding is a dot product with -1 and 0, and exact.)
template <int N> __device__ __forceinline__ void split(const float *x, bf16x8_t *parts) {
    uint32_t first = 0x0000bf80u, second = 0xbf800000u;  // (-1, 0), (0, -1): in registers, since
    asm("" : "+s"(first), "+s"(second));  // as constants of the instruction they are read otherwise
    uint32_t p[N][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float u = x[2 * i], v = x[2 * i + 1];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            p[n][i] = pack2(u, v);
            if (n == N - 1) break;
            const bf16x2_t r = __builtin_bit_cast(bf16x2_t, p[n][i]);
            u = __builtin_amdgcn_fdot2_f32_bf16(r, __builtin_bit_cast(bf16x2_t, first), u, false);
            v = __builtin_amdgcn_fdot2_f32_bf16(r, __builtin_bit_cast(bf16x2_t, second), v, false);
        }
    }
#pragma unroll
    for (int n = 0; n < N; ++n) parts[n] = __builtin_bit_cast(bf16x8_t, make_uint4(p[n][0], p[n][1], p[n][2], p[n][3]));
}
__device__ __forceinline__ void split(const f32x8_t &x, bf16x8x3_t &f) {
    const float z[8] = {x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]};
    split<3>(z, f.p);
}

// Values 8a .. 8a + 7 of a result as the operand of a step over its rows 16a .. 16a + 15.
// A weight rounded to bfloat16 once is off by up to 2^-8, as much again as the rounding of a
// stored output: beside bfloat16 values weights go in two parts, good to 2^-16.
template <typename S> struct Weights;
template <> struct Weights<uint16_t> {
    bf16x8_t p[2];
    __device__ __forceinline__ Weights(const f32x16_t &x, int a) {
        float z[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = x[8 * a + i];
        split<2>(z, p);
    }
    __device__ __forceinline__ f32x16_t add(const bf16x8_t &f, const f32x16_t &c) const {
        return mma(f, p[0], mma(f, p[1], c));
    }
};
template <> struct Weights<float> {
    bf16x8x3_t w;
    __device__ __forceinline__ Weights(const f32x16_t &x, int a) {
        float z[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = x[8 * a + i];
        split<3>(z, w.p);
    }
    __device__ __forceinline__ f32x16_t add(const bf16x8x3_t &f, const f32x16_t &c) const { return mma(f, w, c); }
};
template <> struct Weights<whole_t> {
    f32x8_t w;
    __device__ __forceinline__ Weights(const f32x16_t &x, int a) {
#pragma unroll
        for (int s = 0; s < 8; ++s) w[s] = x[8 * a + s];
    }
    __device__ __forceinline__ f32x16_t add(const f32x8_t &f, const f32x16_t &c) const { return mma(f, w, c); }
};

// The other half's value of the same row (lanes l and l ^ 32) joined with the lane's own.
__device__ __forceinline__ float half_max(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ __forceinline__ float ex2(float x) { return __builtin_amdgcn_exp2f(x); }

// Waits until at most N of this wave's vector-memory operations are outstanding; no access to
// memory moves across.  (The builtin, so that the compiler knows its own loads done.)
template <int N> __device__ __forceinline__ void wait_loads() {
    __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | ((N >> 4) << 14));
    asm volatile("" : : : "memory");
}
// Waits until this wave's reads of LDS are done.
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory"); }

__device__ __forceinline__ uint32_t lds_address(const void *p) {
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char *)p;
}

// A value that is the same in every lane.
__device__ __forceinline__ uint32_t uniform(uint64_t x) {
    return (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)x);
}

// The buffer loads that write LDS directly: each lane's 4 or 16 bytes at byte `off` of the
// buffer go to LDS byte `to` (the same in every lane) + the lane's place; past the buffer's end
// zeros do.  Written in assembly, without a register loaded, so that reads of other LDS do not
// wait for them: their own readers do so by wait_loads and, across waves, a barrier.  s_nop 4:
// the wait states between a vector write of a scalar register (a spilled one restored, say) and
// its use by a load; s_nop 0: between m0 and a load to LDS.  m0 is named as written, so that no
// setting of it is kept across them (that it is a register the compiler reserves is what it
// would warn of).
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_lds4(uint32_t to, u32x4_t buf, int off) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dword %1, %2, 0 offen lds"
                 :
                 : "s"(to), "v"(off), "s"(buf)
                 : "memory", "m0");
}
__device__ __forceinline__ void load_lds16(uint32_t to, u32x4_t buf, int off) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 :
                 : "s"(to), "v"(off), "s"(buf)
                 : "memory", "m0");
}
// Four of them, `step` bytes of LDS apart.
__device__ __forceinline__ void load_lds16(uint32_t to, uint32_t step, u32x4_t buf, const int *off) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %2, %6, 0 offen lds\n\t"
                 "s_add_u32 m0, m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %3, %6, 0 offen lds\n\t"
                 "s_add_u32 m0, m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %4, %6, 0 offen lds\n\t"
                 "s_add_u32 m0, m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %5, %6, 0 offen lds"
                 :
                 : "s"(to), "s"(step), "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "s"(buf)
                 : "memory", "m0", "scc");
}
#pragma clang diagnostic pop
__device__ __forceinline__ u32x4_t buffer_of(const void *src, uint32_t bytes) {
    const uint64_t base = (uint64_t)src;
    return u32x4_t{uniform(base), uniform((base >> 32) & 0xffffu), uniform(bytes), 0x00027000u};
}

// Rows of D values staged in LDS: row-major, the 16-byte chunks of a row exchanged by an XOR
// with swz(row).  LDS serves 64 banks of 4 bytes a cycle: 16 lanes' chunks of 16 consecutive
// rows (row_frag) and 64 bytes of each of 4 consecutive bfloat16 rows (operand_t) fall on
// different banks.  bfloat16 rows of 128 values, 256 bytes, do so by an XOR within four rows
// and 16 bytes between fours, which takes fewer addresses than an XOR alone.  Float32 rows
// share some banks: their products, not their reads, take the time.
template <typename S, int D> struct Tile {
    static constexpr int kRow = D * (int)sizeof(S);  // bytes of a row
    static constexpr int kChunks = kRow / 16;
    static constexpr int kRowsPerLoad = 1024 / kRow;  // rows a wave moves per instruction
    static constexpr int kBlock = 1024 + (sizeof(S) == 2 && kChunks == 16 ? 16 : 0);  // bytes they take

    static constexpr int bytes(int rows) { return rows / kRowsPerLoad * kBlock; }

    __device__ __forceinline__ static int swz(int row) {
        if (kChunks == 4) return (row >> 2) & 3;
        if (kChunks == 8) return ((row & 2) << 1) | ((row & 4) >> 1) | ((row >> 3) & 1);
        if (sizeof(S) == 2) return (row & 3) << 2;
        return ((row & 1) << 2) | (row & 2) | ((row >> 2) & 1);
    }
    // Chunk ch of a staged row.
    __device__ __forceinline__ static const char *at(const char *t, int row, int ch) {
        return t + row / kRowsPerLoad * kBlock + row % kRowsPerLoad * kRow + 16 * (ch ^ swz(row));
    }

    // Rows [0, N) at `src`, `stride` bytes apart (64 of them below 2^31 bytes), to `dst` by the
    // buffer loads that write LDS directly.  Rows from `valid` (>= 1) on are read past the
    // buffer's end and come back as zeros: a weight of 0 never meets an infinity there.  LAST: they
    // repeat the last valid row, which has no product that this one has not (a zero has: with
    // an infinity, a NaN).  The loads are shared by NW waves; this is wave w.
    template <int N, int NW, bool LAST = false>
    __device__ __forceinline__ static void stage(char *dst, const char *src, long long stride, int valid, int w) {
        constexpr int loads = N / kRowsPerLoad, each = (loads + NW - 1) / NW;
        const int lane = threadIdx.x & 63;
        const int rr = lane / kChunks, pc = lane % kChunks;
        const int st = (int)stride;
        const u32x4_t buf = buffer_of(src, (uint32_t)((min(valid, N) - 1) * st + kRow));
        const uint32_t to = uniform(lds_address(dst) + kBlock * w);
        int off[each];
#pragma unroll
        for (int a = 0; a < each; ++a) {
            const int r = (a * NW + w) * kRowsPerLoad + rr;
            off[a] = r < valid || LAST ? min(r, valid - 1) * st + 16 * (pc ^ swz(r)) : 0x7fffff00;
        }
        if constexpr (each % 4 == 0) {
#pragma unroll
            for (int a = 0; a < each; a += 4) load_lds16(to + kBlock * NW * a, kBlock * NW, buf, off + a);
        } else {
#pragma unroll
            for (int a = 0; a < each; ++a)
                if (loads % NW == 0 || a * NW + w < loads) load_lds16(to + kBlock * NW * a, buf, off[a]);
        }
    }

    // Row `row`, step ks: values 16 ks + 8h .. + 7.
    __device__ __forceinline__ static void row_frag(const char *t, int row, int ks, int h, bf16x8_t &f) {
        f = *reinterpret_cast<const bf16x8_t *>(at(t, row, 2 * ks + h));
    }
    __device__ __forceinline__ static void row_frag(const char *t, int row, int ks, int h, f32x8_t &f) {
        const f32x4_t x = *reinterpret_cast<const f32x4_t *>(at(t, row, 4 * ks + 2 * h));
        const f32x4_t y = *reinterpret_cast<const f32x4_t *>(at(t, row, 4 * ks + 2 * h + 1));
        f = f32x8_t{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
    }
    __device__ __forceinline__ static void row_frag(const char *t, int row, int ks, int h, bf16x8x3_t &f) {
        f32x8_t x;
        row_frag(t, row, ks, h, x);
        split(x, f);
    }

    // Column 32 dt + l % 32 of the 16 rows from r0 (a multiple of 16), in the order of a
    // result's rows: 4h .. 4h + 3, 8 + 4h .. 8 + 4h + 3.  bfloat16: two LDS transpose reads;
    // in each group of 16 lanes lane m points at 4 values (8 bytes) of row m / 4, and lane n
    // receives value n % 4 of the pieces of lanes n / 4, n / 4 + 4, n / 4 + 8, n / 4 + 12.
    __device__ __forceinline__ static void operand_t(const char *t, int r0, int dt, bf16x8_t &f) {
        const int lane = threadIdx.x & 63, h = lane >> 5, m = lane & 15;
        const int ch = 4 * dt + 2 * ((lane >> 4) & 1) + ((m & 3) >> 1);
        i16x4_t x[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int r = r0 + 8 * j + 4 * h + (m >> 2);
            x[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) i16x4_t *)(at(t, r, ch) + 8 * (m & 1)));
        }
        f = __builtin_bit_cast(bf16x8_t, x);
    }
    __device__ __forceinline__ static void operand_t(const char *t, int r0, int dt, f32x8_t &f) {
        const int lane = threadIdx.x & 63, h = lane >> 5, d = 32 * dt + (lane & 31);
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            const int r = r0 + 8 * (s >> 2) + 4 * h + (s & 3);
            f[s] = *reinterpret_cast<const float *>(at(t, r, d >> 2) + 4 * (d & 3));
        }
    }
    __device__ __forceinline__ static void operand_t(const char *t, int r0, int dt, bf16x8x3_t &f) {
        f32x8_t x;
        operand_t(t, r0, dt, x);
        split(x, f);
    }
};

// Step ks of a row in global memory (rows are 16-byte aligned).
__device__ __forceinline__ void load_frag(const uint16_t *row, int ks, int h, bf16x8_t &f) {
    f = *reinterpret_cast<const bf16x8_t *>(row + 16 * ks + 8 * h);
}
__device__ __forceinline__ void load_frag(const float *row, int ks, int h, f32x8_t &f) {
    const f32x4_t *p = reinterpret_cast<const f32x4_t *>(row + 16 * ks + 8 * h);
    f = f32x8_t{p[0][0], p[0][1], p[0][2], p[0][3], p[1][0], p[1][1], p[1][2], p[1][3]};
}
__device__ __forceinline__ void load_frag(const float *row, int ks, int h, bf16x8x3_t &f) {
    f32x8_t x;
    load_frag(row, ks, h, x);
    split(x, f);
}
// Its inner product with the same step of another row.
__device__ __forceinline__ float dot_rows(const uint16_t *a, const uint16_t *b, int ks, int h) {
    float x[8], y[8], s = 0.f;
    Vec<uint16_t>::load(a + 16 * ks + 8 * h, x);
    Vec<uint16_t>::load(b + 16 * ks + 8 * h, y);
#pragma unroll
    for (int j = 0; j < 8; ++j) s = fmaf(x[j], y[j], s);
    return s;
}
__device__ __forceinline__ float dot_rows(const float *a, const float *b, int ks, int h) {
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) s = fmaf(a[16 * ks + 8 * h + j], b[16 * ks + 8 * h + j], s);
    return s;
}

// The inner product of two rows, by one lane.
template <typename S, int D> __device__ __forceinline__ float dot_row(const S *a, const S *b) {
    constexpr int V = 16 / (int)sizeof(S);
    float s = 0.f;
    for (int d = 0; d < D; d += V) {
        float x[V], y[V];
        Vec<S>::load(a + d, x);
        Vec<S>::load(b + d, y);
#pragma unroll
        for (int e = 0; e < V; ++e) s = fmaf(x[e], y[e], s);
    }
    return s;
}
__device__ __forceinline__ float value_of(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ float value_of(float x) { return x; }
__device__ __forceinline__ void put_value(uint16_t *p, float x) { *p = (uint16_t)f32_to_bf16(x); }
__device__ __forceinline__ void put_value(float *p, float x) { *p = x; }

// Stores the lane's column of D / 32 results (column = a row of the output, rows = its
// values) times `scale`.  Both halves of a row must be active.
template <int D>
__device__ __forceinline__ void store_cols(float *row, const f32x16_t *acc, float scale, int h) {
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const f32x4_t x = {acc[dt][4 * j] * scale, acc[dt][4 * j + 1] * scale, acc[dt][4 * j + 2] * scale,
                               acc[dt][4 * j + 3] * scale};
            *reinterpret_cast<f32x4_t *>(row + 32 * dt + 8 * j + 4 * h) = x;
        }
}
template <int D>
__device__ __forceinline__ void store_cols(uint16_t *row, const f32x16_t *acc, float scale, int h) {
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
            // values 8j + 4h .. + 3 and 8 (j + 1) + 4h .. + 3: the halves exchange a piece each,
            // so that half h stores values 8 (j + h) .. + 7 at once
            uint32_t a[2], b[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint32_t x = pack2(acc[dt][4 * j + 2 * e] * scale, acc[dt][4 * j + 2 * e + 1] * scale);
                const uint32_t y = pack2(acc[dt][4 * j + 4 + 2 * e] * scale, acc[dt][4 * j + 5 + 2 * e] * scale);
                const auto r = __builtin_amdgcn_permlane32_swap(x, y, false, false);
                a[e] = r[0];
                b[e] = r[1];
            }
            *reinterpret_cast<uint4 *>(row + 32 * dt + 8 * (j + h)) = make_uint4(a[0], a[1], b[0], b[1]);
        }
}

// One set of states that queries attend to.  A problem is one key/value head of one batch
// entry of the states; its query rows are numbered r = ((b - b0) G + g) T + t over the
// batch entries that read it (all of them where the batch shares the states).
struct States {
    const void *k, *v;
    Layout lk, lv;
    const int *lens;  // valid rows per batch entry of the states; null: S
    int S;
    int share;   // batch entries that read one problem: 1, or B
    int causal;  // query t reads rows [0, len - T + 1 + t) only
    int rows;    // share G T
    int rw;      // 32 rw rows to a workgroup of 8 waves; 0: 32 rows to one of 4
    int tiles;   // row tiles of a problem
    int splits;  // pieces of the states' rows
    int slot;    // first partial result of these states
};

// Sizes of a call and the queries' side.
struct Queries {
    const void *q;
    void *o;
    float *lse;
    Layout lq, lo;
    float *part_o;    // partial results [slot][B H T][D] and their lse [slot][B H T]
    float *part_lse;  // (null: one piece, written to o and lse)
    int B, H, Hkv, G, T;
    float scale;  // tau log2 e
};

// Row r of problem (b0, j): batch entry, query head, position.
struct RowAt {
    int b, h, t;
};
__device__ __forceinline__ RowAt row_at(const Queries &a, int b0, int j, int r) {
    const int hq = r / a.T;
    const int b = hq / a.G;
    return {b0 + b, j * a.G + (hq - b * a.G), r - hq * a.T};
}

__device__ __forceinline__ int states_len(const States &s, int b) {
    return s.lens ? min(max(s.lens[b], 0), s.S) : s.S;
}

// Block index -> work item, consecutive items (the row tiles and pieces of one problem) on
// one XCD, whose L2 then holds the problem's rows: workgroups go round-robin over 8 XCDs.
__device__ __forceinline__ int xcd_item(int b, int n) {
    const int per = n >> 3, rem = n & 7;
    const int x = b & 7, y = b >> 3;
    return x * per + min(x, rem) + y;
}

}  // namespace fibattn
