// Dense attention to states that are not the sequence's own (an encoder's, a memory or a
// prefix that the batch shares): the pieces its kernels share.
//
// Every product runs on 32 x 32 matrix-core tiles.  A tile's operands hold, per lane, 8
// values of one row: lane l serves row l % 32 and the inner indices 8h .. 8h + 7 of a step
// of 16, h = l / 32 (Frag).  bfloat16 takes one v_mfma_f32_32x32x16_bf16 a step, float32
// eight v_mfma_f32_32x32x2_f32 whose slot s pairs inner indices s and 8 + s.  The result
// holds column l % 32 and rows 8 (i / 4) + 4h + i % 4, i < 16.
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
typedef unsigned u32x2_t __attribute__((ext_vector_type(2)));

template <typename S> struct FragOf;
template <> struct FragOf<uint16_t> { typedef bf16x8_t type; };
template <> struct FragOf<float> { typedef f32x8_t type; };
template <typename S> using Frag = typename FragOf<S>::type;

__device__ __forceinline__ f32x16_t mma(const bf16x8_t &a, const bf16x8_t &b, const f32x16_t &c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
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

// Values 8a .. 8a + 7 of a result as the operand of a step over its rows 16a .. 16a + 15.
// bfloat16: each weight is rounded once, by at most 2^-8 of itself, as the stored values
// it multiplies were; the sums stay in float32.
__device__ __forceinline__ void to_frag(const f32x16_t &x, int a, bf16x8_t &f) {
    uint4 u;
    u.x = pack2(x[8 * a], x[8 * a + 1]);
    u.y = pack2(x[8 * a + 2], x[8 * a + 3]);
    u.z = pack2(x[8 * a + 4], x[8 * a + 5]);
    u.w = pack2(x[8 * a + 6], x[8 * a + 7]);
    f = __builtin_bit_cast(bf16x8_t, u);
}
__device__ __forceinline__ void to_frag(const f32x16_t &x, int a, f32x8_t &f) {
#pragma unroll
    for (int s = 0; s < 8; ++s) f[s] = x[8 * a + s];
}

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

// Waits until at most N of this wave's vector-memory operations are outstanding.
template <int N> __device__ __forceinline__ void wait_loads() {
    __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | ((N >> 4) << 14));
}

// Rows of D values staged in LDS: row-major, the 16-byte chunks of a row exchanged by an XOR
// with swz(row).  Reading one chunk of 8 consecutive rows (row_frag) then touches every bank
// once, and so do the transposed reads, which take 64 bytes of each of 4 consecutive rows.
template <typename S, int D> struct Tile {
    static constexpr int kRow = D * (int)sizeof(S);  // bytes of a row
    static constexpr int kChunks = kRow / 16;
    static constexpr int kRowsPerLoad = 1024 / kRow;  // rows a wave moves per instruction

    __device__ __forceinline__ static int swz(int row) {
        if (kChunks == 4) return (row >> 1) & 3;
        return ((row & 1) << 2) | (row & 2) | ((row >> 2) & 1);
    }

    // Rows [0, N) at `src`, `stride` bytes apart (64 of them below 2^31 bytes), to `dst` by the
    // buffer loads that write LDS directly.  Rows from `valid` (>= 1) on are read past the buffer's
    // end and come back as zeros: a weight of 0 never meets an infinity there.  The loads are
    // shared by NW waves; this is wave w.
    template <int N, int NW>
    __device__ __forceinline__ static void stage(char *dst, const char *src, long long stride, int valid, int w) {
        constexpr int loads = N / kRowsPerLoad;
        const int lane = threadIdx.x & 63;
        const int rr = lane / kChunks, pc = lane % kChunks;
        const int st = (int)stride;
        const __amdgpu_buffer_rsrc_t buf =
            __builtin_amdgcn_make_buffer_rsrc((void *)src, 0, (min(valid, N) - 1) * st + kRow, 0x00027000);
#pragma unroll
        for (int a = 0; a < (loads + NW - 1) / NW; ++a) {
            const int blk = a * NW + w;
            if (loads % NW && blk >= loads) break;
            const int r = blk * kRowsPerLoad + rr;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (__attribute__((address_space(3))) void *)(dst + 1024 * blk), 16,
                                                     r < valid ? r * st + 16 * (pc ^ swz(r)) : 0x7fffff00, 0, 0, 0);
        }
    }

    // Row `row`, step ks: values 16 ks + 8h .. + 7.
    __device__ __forceinline__ static void row_frag(const char *t, int row, int ks, int h, bf16x8_t &f) {
        f = *reinterpret_cast<const bf16x8_t *>(t + row * kRow + 16 * ((2 * ks + h) ^ swz(row)));
    }
    __device__ __forceinline__ static void row_frag(const char *t, int row, int ks, int h, f32x8_t &f) {
        const f32x4_t x = *reinterpret_cast<const f32x4_t *>(t + row * kRow + 16 * ((4 * ks + 2 * h) ^ swz(row)));
        const f32x4_t y = *reinterpret_cast<const f32x4_t *>(t + row * kRow + 16 * ((4 * ks + 2 * h + 1) ^ swz(row)));
        f = f32x8_t{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
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
                (__attribute__((address_space(3))) i16x4_t *)(t + r * kRow + 16 * (ch ^ swz(r)) + 8 * (m & 1)));
        }
        f = __builtin_bit_cast(bf16x8_t, x);
    }
    __device__ __forceinline__ static void operand_t(const char *t, int r0, int dt, f32x8_t &f) {
        const int lane = threadIdx.x & 63, h = lane >> 5, d = 32 * dt + (lane & 31);
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            const int r = r0 + 8 * (s >> 2) + 4 * h + (s & 3);
            f[s] = *reinterpret_cast<const float *>(t + r * kRow + 16 * ((d >> 2) ^ swz(r)) + 4 * (d & 3));
        }
    }
};

// Step ks of a row in global memory (rows are 16-byte aligned).
__device__ __forceinline__ void load_frag(const uint16_t *row, int ks, int h, bf16x8_t &f) {
    f = *reinterpret_cast<const bf16x8_t *>(row + 16 * ks + 8 * h);
}
__device__ __forceinline__ void load_frag(const float *row, int ks, int h, f32x8_t &f) {
    f = *reinterpret_cast<const f32x8_t *>(row + 16 * ks + 8 * h);
}
__device__ __forceinline__ float dot_frag(const bf16x8_t &a, const bf16x8_t &b) {
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) s = fmaf((float)a[j], (float)b[j], s);
    return s;
}
__device__ __forceinline__ float dot_frag(const f32x8_t &a, const f32x8_t &b) {
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) s = fmaf(a[j], b[j], s);
    return s;
}

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
