// Int8 dense layers whose inputs are quantised with a scale for each token (row) and whose weights have one for each channel:
//   s_x[m] = max_k |x[m,k]| / 127,  q[m,k] = rint(x[m,k] * 127 / max),  y[m,n] = (sum_k q[m,k] w[n,k]) s_x[m] s_w[n] + b[n].
//
// Both operands lie packed in the order in which the matrix instruction takes them: tiles of 16 rows x 64 bytes of K,
// [row tile][k step][lane = 16 * (k % 64 / 16) + row % 16][16 bytes], K padded with zeros to whole pairs of steps.  A tile is one
// contiguous KiB, so every operand load is one coalesced access, goes to LDS without passing registers, and is read back from there
// without bank conflicts; no kernel meets a K that ends inside a step.  Features are the matrix instruction's rows: a lane ends up
// with four consecutive features of one token.
#include <stdio.h>

#include <type_traits>

#include "wide_ops.h"

namespace accerl {

int conv_num_cus();   // compute units of the current device

namespace {

constexpr int64_t DI_MAX_ROWS = 1 << 24, DI_MAX_K = 1 << 16;      // 2^16 * 128 * 128 is half of what an int32 sum holds

__host__ __device__ inline int64_t di_steps(int64_t K) { return (K + 127) / 128 * 2; }

// ---------------------------------------------------------------- quantising
// Sixteen elements of a row as they lie in memory.
template <typename T> struct Piece { u32x4 w[sizeof(T)]; };

template <typename T>
__device__ __forceinline__ void piece_load(Piece<T>& d, const T* row, int64_t k, int64_t cols) {
    if (k + 16 <= cols) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T); ++i) {
            if constexpr (sizeof(T) == 4) d.w[i] = *(const u32x4_at4*)((const char*)(row + k) + 16 * i);
            else d.w[i] = *(const u32x4_at2*)((const char*)(row + k) + 16 * i);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < (int)sizeof(T); ++i) d.w[i] = (u32x4){0, 0, 0, 0};
    if (k >= cols) return;
#pragma unroll
    for (int e = 0; e < 16; ++e)
        if (k + e < cols) {
            const uint32_t u = sizeof(T) == 4 ? ((const uint32_t*)row)[k + e] : (uint32_t)((const uint16_t*)row)[k + e];
            constexpr int PER = 4 / (int)sizeof(T);
            d.w[e / (4 * PER)][e / PER % 4] |= u << (16 * (e % PER));
        }
}
// Magnitudes are compared as integers, in which a NaN is larger than everything; 16-bit elements two at a time.
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
template <typename T>
__device__ __forceinline__ void piece_max(const Piece<T>& d, uint32_t& m) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T); ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (sizeof(T) == 4) m = max(m, d.w[i][e] & 0x7fffffffu);
            else m = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, m), __builtin_bit_cast(u16x2, d.w[i][e] & 0x7fff7fffu)));
        }
}
template <typename T>
__device__ __forceinline__ void piece_floats(const Piece<T>& d, float (&v)[16]) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T); ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (sizeof(T) == 4) v[4 * i + e] = __uint_as_float(d.w[i][e]);
            else el_pair<T>(d.w[i][e], v[8 * i + 2 * e], v[8 * i + 2 * e + 1]);
        }
}

// Rounded once, from the exact quotient: the product with 1 / max is off by a few parts in 2^24, so the candidate it gives may lie on the
// wrong side of the middle of two steps; the remainder x * 127 - q * max is exact (in 32 bits for 8- and 11-bit significands, in
// 64 for fp32) and tells the side.  Ties go to the even step.
template <typename T>
__device__ __forceinline__ int di_quant(float x, float inv, float top) {
    float q = rintf(x * inv);
    if constexpr (__is_same(T, float)) {
        const double r = fma(-(double)q, (double)top, (double)x * 127.0), two = 2.0 * fabs(r);
        if (two > (double)top || (two == (double)top && ((int)q & 1))) q += r > 0.0 ? 1.0f : -1.0f;
    } else {
        const float r = fmaf(-q, top, x * 127.0f), two = 2.0f * fabsf(r);
        if (two > top || (two == top && ((int)q & 1))) q += r > 0.0f ? 1.0f : -1.0f;
    }
    return (int)q;
}
// the power of two by which a row is scaled where 127 / max or 127 * x would leave the range
__device__ __forceinline__ float di_by(float top) { return top < 0x1p-100f ? 0x1p100f : top > 0x1p100f ? 0x1p-20f : 1.0f; }
// Sixteen of them.  x * inv + 1.5 * 2^23 has the rounded quotient in its low byte; only where one of the sixteen lies within 2^-15 of the
// middle of two steps (inv's error moves a quotient by less than 2^-16), or the row's magnitude needs scaling, are they looked at one by
// one.  That is 5 operations an element in place of 15: 8192 rows of 4096 bf16 were bound by them (31 us).
template <typename T>
__device__ __forceinline__ v4i di_quant16(const Piece<T>& d, float inv, float top, float by) {
    constexpr float MAGIC = 12582912.0f;
    float v[16], off = 0.0f;
    uint32_t u[16];
    piece_floats(d, v);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const float q = fmaf(v[e], inv, MAGIC);
        off = fmaxf(off, fabsf(fmaf(v[e], inv, MAGIC - q)));
        u[e] = __float_as_uint(q);
    }
    if (off > 0.5f - 0x1p-15f || by != 1.0f) {
#pragma unroll
        for (int e = 0; e < 16; ++e) u[e] = (uint32_t)di_quant<T>(v[e] * by, inv, top);
    }
    v4i o;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        o[k] = (int)__builtin_amdgcn_perm(__builtin_amdgcn_perm(u[4 * k + 3], u[4 * k + 2], 0x0c0c0400), __builtin_amdgcn_perm(u[4 * k + 1], u[4 * k], 0x0c0c0400), 0x05040100);
    return o;
}

// A workgroup quantises ROWS rows: lane l of a wavefront is row l % ROWS and one of 64 / ROWS pieces of 16 elements, so that a wavefront
// reads runs of consecutive elements and writes runs of 16 ROWS bytes.  What a lane reads for the maximum stays in registers
// (HOLD pieces; longer rows read the rest again).  A row that holds a NaN or an infinity gets it as its scale and zeros, so that its
// results are NaN.
constexpr int QR_THREADS = 256;
// One row a workgroup up to 1024 rows (1024 x 4096 bf16 7.5 us, four rows 9.9; 2048 x 1024 6.7 / 4.7), 16 where a row is one pass of its 16
// lanes (16384 x 256 6.0, four 9.3; 4096 x 512 6.3 / 4.9).  8192 x 4096 bf16 takes 23.5 us, 4.1 TB/s.
constexpr int64_t QR_SINGLE = 1024, QR_SHORT = 256;
template <typename T, int ROWS, int HOLD>
__global__ __launch_bounds__(QR_THREADS) void quantize_rows_kernel(const T* x, int64_t rows, int64_t cols, int64_t ld, v4i* out, float* scale, int steps) {
    constexpr int LANES = QR_THREADS / ROWS;                        // lanes a row
    __shared__ uint32_t s_max[QR_THREADS / 64][ROWS];
    const int tid = threadIdx.x, r = tid % ROWS, piece = tid / ROWS;
    const int64_t row = (int64_t)blockIdx.x * ROWS + r;
    const bool real = row < rows;                                   // the rows that fill the last tile are zeros
    const T* src = x + (real ? row : rows - 1) * ld;
    Piece<T> v[HOLD], w;
    uint32_t m = 0;
#pragma unroll
    for (int h = 0; h < HOLD; ++h) piece_load(v[h], src, (int64_t)(piece + h * LANES) * 16, cols);
#pragma unroll
    for (int h = 0; h < HOLD; ++h) piece_max(v[h], m);
    for (int64_t k = (int64_t)(piece + HOLD * LANES) * 16; k < cols; k += LANES * 16) {
        piece_load(w, src, k, cols);
        piece_max(w, m);
    }
    if constexpr (sizeof(T) == 2) m = max(m & 0xffffu, m >> 16);
#pragma unroll
    for (int o = ROWS; o < 64; o <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o));
    if ((tid & 63) < ROWS) s_max[tid >> 6][r] = m;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < QR_THREADS / 64; ++k) m = max(m, s_max[k][r]);
    float top;
    if constexpr (sizeof(T) == 4) top = __uint_as_float(m);
    else { T t; t.u = (uint16_t)m; top = el_f32(t); }
    if (real && piece == 0) scale[row] = top / 127.0f;
    const float by = di_by(top);
    const bool zero = !real || !(top > 0.0f && __float_as_uint(top) < 0x7f800000u);
    top *= by;
    const float inv = 127.0f / top;
    v4i* dst = out + (row >> 4) * steps * 64 + (row & 15);
#pragma unroll
    for (int h = 0; h < HOLD; ++h) {
        const int p = piece + h * LANES;
        if (p < steps * 4) dst[p * 16] = zero ? (v4i){0, 0, 0, 0} : di_quant16<T>(v[h], inv, top, by);
    }
    for (int p = piece + HOLD * LANES; p < steps * 4; p += LANES) {
        piece_load(w, src, (int64_t)p * 16, cols);
        dst[p * 16] = zero ? (v4i){0, 0, 0, 0} : di_quant16<T>(w, inv, top, by);
    }
}

// int8 rows to tiles and back, a 16-byte piece a thread: with every update of int8 weights.  Bound by its byte loads and stores: 16384 x 4096 116 us
// (back 120), 1.2 TB/s; 2501 x 1777 8.9 (12.8).
__global__ __launch_bounds__(256) void pack_rows_kernel(const int8_t* q, int64_t rows, int64_t cols, int64_t ld, v4i* out, int64_t steps, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t tile = i / (steps * 64), p = i - tile * steps * 64, row = tile * 16 + (p & 15), k = (p >> 4) * 16;
        union { v4i v; int8_t b[16]; } u;
#pragma unroll
        for (int e = 0; e < 16; ++e) u.b[e] = row < rows && k + e < cols ? q[row * ld + k + e] : 0;
        out[i] = u.v;
    }
}
__global__ __launch_bounds__(256) void unpack_rows_kernel(const v4i* in, int64_t rows, int64_t cols, int64_t ld, int8_t* q, int64_t steps, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t tile = i / (steps * 64), p = i - tile * steps * 64, row = tile * 16 + (p & 15), k = (p >> 4) * 16;
        union { v4i v; int8_t b[16]; } u;
        u.v = in[i];
        if (row < rows)
            for (int e = 0; e < 16 && k + e < cols; ++e) q[row * ld + k + e] = u.b[e];
    }
}

// ---------------------------------------------------------------- the product
struct DenseParams {
    const char* x;           // packed tokens
    const char* w;           // packed features
    const float* sx;
    const float* sw;
    const float* bias;       // NULL = none
    void* out;
    int64_t M, N, ld;        // tokens, features, elements between output rows
    int xt, wt, steps;       // row tiles of either operand, matrix steps (even)
    int dtype, relu;
};

__device__ __forceinline__ float di_result(const DenseParams& p, int acc, float sx, float sw, float b) {
    const float y = fmaf((float)acc * sx, sw, b);
    return p.relu && y < 0.0f ? 0.0f : y;                         // a NaN stays
}
// results of features n .. n + 3 of token m
template <typename T>
__device__ __forceinline__ void di_store(const DenseParams& p, const v4i& acc, int64_t m, int64_t n, float sx, const float (&sw)[4], const float (&b)[4]) {
    float y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = di_result(p, acc[e], sx, sw[e], b[e]);
    T* o = (T*)p.out + m * p.ld + n;
    if (n + 4 <= p.N) {
        if constexpr (__is_same(T, float)) {
            typedef v4f v4f_at4 __attribute__((aligned(4)));
            *(v4f_at4*)o = (v4f){y[0], y[1], y[2], y[3]};
        } else {
            *(u32x2_at2*)o = (u32x2){f32_pair<T>(y[0], y[1]), f32_pair<T>(y[2], y[3])};
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) if (n + e < p.N) o[e] = f32_el<T>(y[e]);
    }
}
__device__ __forceinline__ void di_channels(const DenseParams& p, int64_t n, float (&sw)[4], float (&b)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int64_t i = min(n + e, p.N - 1);
        sw[e] = p.sw[i];
        b[e] = p.bias ? p.bias[i] : 0.0f;
    }
}

// Large products.  A workgroup of WF x WT wavefronts owns (16 WF FA) features x (16 WT FB) tokens.  Of a step (64 bytes of every row) the
// features, which WT wavefronts share, go from memory to registers three steps ahead, to one of three LDS buffers one step ahead, and to the
// registers of the fragments that they replace between the matrix instructions of the step before; the tokens go to registers
// straight from memory, two steps ahead.  (Both through LDS, a workgroup of 256 x 256 moves 128 KiB a step through it, which takes as
// long as the step's matrix instructions; like this 80 KiB, and 48 KiB through the first-level cache.)  One barrier a step.
// 8192 x 4096 x 16384 429 us, 2.56 POP/s; its matrix instructions alone, from registers, with random data, would take 271 (4.05 POP/s, where
// the card's power ends it; zeros 4.8).  A tile's results, about 11 us of a round, overlap no other tile's steps.
//
// LDS operations of a wavefront end in their order.  In step t - 1 a wavefront writes its fragments of step t + 1, then reads those of step t:
// where no more than FA operations are outstanding, reads of step t - 1 all of them, its writes of step t + 1 and its reads of step
// t - 1 (issued in step t - 2) are done.  When everybody has passed the barrier of step t like that, step t + 1 can be read and the buffer
// of step t - 1 filled again.
template <typename T, int WF, int WT, int FA, int FB, int KS>
__global__ __launch_bounds__(64 * WF * WT, 2) void dense_i8_tile_kernel(const DenseParams p) {
    constexpr int WAVES = WF * WT, BF = WF * FA, BT = WT * FB;      // row tiles of a workgroup
    constexpr int PA = BF * KS / WAVES, BUF = BF * KS * 1024;       // fragments of features a wavefront brings per stage of KS steps
    static_assert(BF * KS % WAVES == 0 && FA * KS < 16, "whole fragments a wavefront; the count of outstanding operations has four bits");
    // results on their way out: 16 tokens x 16 CH features of a wavefront, rows 16 bytes apart
    constexpr int CH = FA * 256 * (int)sizeof(T) <= 4096 ? FA : 16 / (int)sizeof(T), ROW = CH * 16 * (int)sizeof(T), PITCH = ROW + 16;
    constexpr int OUT = WAVES * 16 * PITCH, LDS = 3 * BUF > OUT ? 3 * BUF : OUT;
    __shared__ __attribute__((aligned(16))) char s_buf[LDS];
    __shared__ __attribute__((aligned(16))) float s_sw[BF * 16], s_bias[BF * 16], s_sx[BT * 16];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wf = wave % WF, wt = wave / WF;

    // Workgroup n runs on XCD n mod 8.  Every XCD takes consecutive tiles of an order that walks bands of four tiles of tokens, so that
    // the workgroups that run together on it share rows in its cache.
    const unsigned gf = (p.wt + BF - 1) / BF, gt = (p.xt + BT - 1) / BT, n = gf * gt, id = blockIdx.x, xcd = id & 7;
    const unsigned t = xcd * (n >> 3) + min(xcd, n & 7) + (id >> 3);
    constexpr unsigned GROUP = 4;
    const unsigned band = t / (GROUP * gf), first = band * GROUP, high = min(GROUP, gt - first), in = t - band * GROUP * gf;
    const int tf = (int)(in / high) * BF, tt = (int)(first + in % high) * BT;

    // a tile past the end re-reads the last one, a step past the end the last step; neither is used
    const int stages = p.steps / KS;
    const uint32_t l16 = lane * 16;
    const char *pa[PA], *pb[FB];
#pragma unroll
    for (int i = 0; i < PA; ++i) pa[i] = p.w + ((int64_t)min(tf + (wave * PA + i) / KS, p.wt - 1) * p.steps + (wave * PA + i) % KS) * 1024;
#pragma unroll
    for (int j = 0; j < FB; ++j) pb[j] = p.x + (int64_t)min(tt + wt * FB + j, p.xt - 1) * p.steps * 1024;
    v4i r[3][PA], b[3][FB * KS], a[FA * KS], acc[FA][FB];
    auto load_a = [&](v4i (&d)[PA], int s) {
        const uint32_t at = min(s, stages - 1) * (KS * 1024) + l16;
#pragma unroll
        for (int i = 0; i < PA; ++i) d[i] = *(const v4i*)(pa[i] + at);
    };
    auto load_b = [&](v4i (&d)[FB * KS], int s) {
        const uint32_t at = min(s, stages - 1) * (KS * 1024) + l16;
#pragma unroll
        for (int j = 0; j < FB * KS; ++j) d[j] = *(const v4i*)(pb[j % FB] + at + j / FB * 1024);
    };
    auto write_a = [&](const v4i (&d)[PA], int buf) {
#pragma unroll
        for (int i = 0; i < PA; ++i) *(v4i*)(s_buf + buf * BUF + (wave * PA + i) * 1024 + l16) = d[i];
    };
    load_a(r[0], 0);
    load_b(b[0], 0);
    load_a(r[1], 1);
    load_b(b[1], 1);
    load_a(r[2], 2);
    for (int i = tid; i < BF * 16; i += 64 * WAVES) {
        const int64_t f = min((int64_t)tf * 16 + i, p.N - 1);
        s_sw[i] = p.sw[f];
        s_bias[i] = p.bias ? p.bias[f] : 0.0f;
    }
    for (int i = tid; i < BT * 16; i += 64 * WAVES) s_sx[i] = p.sx[min((int64_t)tt * 16 + i, p.M - 1)];
#pragma unroll
    for (int i = 0; i < FA; ++i)
#pragma unroll
        for (int j = 0; j < FB; ++j) acc[i][j] = (v4i){0, 0, 0, 0};
    write_a(r[0], 0);
    load_a(r[0], 3);
    write_a(r[1], 1);
    load_a(r[1], 4);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < FA * KS; ++i) a[i] = *(const v4i*)(s_buf + ((wf * FA + i % FA) * KS + i / FA) * 1024 + l16);

    auto step = [&](int s, auto C) {
        constexpr int c = decltype(C)::value, c1 = (c + 1) % 3, c2 = (c + 2) % 3;      // c = s % 3
        asm volatile("s_waitcnt lgkmcnt(%0)\n\ts_barrier" ::"n"(FA * KS) : "memory");
        write_a(r[c2], c2);                                                           // step s + 2
        asm volatile("" ::: "memory");                                                // (the barriers count on writes before reads)
        load_a(r[c2], s + 5);
        load_b(b[c2], s + 2);
#pragma unroll
        for (int i = 0; i < FA * KS; ++i) {
#pragma unroll
            for (int j = 0; j < FB; ++j) acc[i % FA][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[i], b[c][i / FA * FB + j], acc[i % FA][j], 0, 0, 0);
            a[i] = *(const v4i*)(s_buf + c1 * BUF + ((wf * FA + i % FA) * KS + i / FA) * 1024 + l16);
        }
        // in this order: writes and the features' loads a matrix instruction apart, then a read and a load behind every row of matrix instructions
#pragma unroll
        for (int i = 0; i < PA; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);
        }
#pragma unroll
        for (int i = 0; i < PA; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
        }
#pragma unroll
        for (int i = 0; i < FA * KS; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, FB, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            if (i * FB / FA < FB * KS) __builtin_amdgcn_sched_group_barrier(0x020, (FB + FA - 1) / FA, 0);
        }
    };
    int s = 0;
    for (; s + 3 <= stages; s += 3) {
        step(s, std::integral_constant<int, 0>());
        step(s + 1, std::integral_constant<int, 1>());
        step(s + 2, std::integral_constant<int, 2>());
    }
    if (s < stages) step(s, std::integral_constant<int, 0>());
    if (s + 1 < stages) step(s + 1, std::integral_constant<int, 1>());

    // A lane's results are four features of a token, 16 tokens an instruction: written like that, a store covers a quarter of a line of 16
    // rows.  They go through LDS, a wavefront's own part of it, and out in pieces of 16 bytes of consecutive features.
    __syncthreads();
    // Whole lines pass the caches by (8192 x 1024 x 16384 186 -> 144 us, 8192 x 4096 x 16384 446 -> 429); rows that do not start with a line would
    // be written in parts of lines (6000 x 2000 x 5000 60.6 -> 64.4).
    const bool past = (((uintptr_t)p.out | (uintptr_t)(p.ld * (int64_t)sizeof(T))) & 127) == 0;
    char* own = s_buf + wave * 16 * PITCH;
    constexpr int EL = 16 / (int)sizeof(T), LANES = ROW / 16, ROWS = 64 / LANES;      // elements of a piece, lanes a row, rows a store
#pragma unroll
    for (int j = 0; j < FB; ++j) {
        const float sx = s_sx[(wt * FB + j) * 16 + (lane & 15)];
        const int64_t m0 = (int64_t)(tt + wt * FB + j) * 16;
#pragma unroll
        for (int i0 = 0; i0 < FA; i0 += CH) {
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                const int f = (wf * FA + i0 + i) * 16 + (lane >> 4) * 4;
                const v4f sw = *(const v4f*)(s_sw + f), bias = *(const v4f*)(s_bias + f);
                float y[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = di_result(p, acc[i0 + i][j][e], sx, sw[e], bias[e]);
                char* to = own + (lane & 15) * PITCH + (i * 16 + (lane >> 4) * 4) * (int)sizeof(T);
                if constexpr (__is_same(T, float)) *(v4f*)to = (v4f){y[0], y[1], y[2], y[3]};
                else *(u32x2*)to = (u32x2){f32_pair<T>(y[0], y[1]), f32_pair<T>(y[2], y[3])};
            }
            const int64_t f = (int64_t)(tf + wf * FA + i0) * 16 + (lane % LANES) * EL;
#pragma unroll
            for (int k = 0; k < 16 / ROWS; ++k) {
                const int64_t m = m0 + k * ROWS + lane / LANES;
                const u32x4 v = *(const u32x4*)(own + (k * ROWS + lane / LANES) * PITCH + (lane % LANES) * 16);
                if (m < p.M && f < p.N) {
                    T* o = (T*)p.out + m * p.ld + f;
                    if (f + EL <= p.N) {
                        if constexpr (__is_same(T, float)) { if (past) __builtin_nontemporal_store(v, (u32x4_at4*)o); else *(u32x4_at4*)o = v; }
                        else { if (past) __builtin_nontemporal_store(v, (u32x4_at2*)o); else *(u32x4_at2*)o = v; }
                    } else {
                        T part[EL];
                        __builtin_memcpy(part, &v, 16);
#pragma unroll
                        for (int e = 0; e < EL; ++e) if (f + e < p.N) o[e] = part[e];
                    }
                }
            }
        }
    }
}

// Few tokens or few tiles: the eight wavefronts of a workgroup split K, each multiplies straight from memory (a weight is read once, by
// one wavefront), and their sums meet in LDS.  Bound by latency: 24 x 2048 x 8192 5.3 us (17 MB of weights at 3.2 TB/s), 301 x 3136 x 512 5.6.
constexpr int KS_WAVES = 8, KS_AHEAD = 8;     // fragments a wavefront has on their way
template <typename T, int FT, int TT>
__global__ __launch_bounds__(64 * KS_WAVES) void dense_i8_ksplit_kernel(const DenseParams p) {
    __shared__ v4i s_acc[KS_WAVES][FT * TT][64];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int tf = blockIdx.x * FT, tt = blockIdx.y * TT;
    const int first = (int)((int64_t)wave * p.steps / KS_WAVES), last = (int)((int64_t)(wave + 1) * p.steps / KS_WAVES);
    const char *pw[FT], *px[TT];
#pragma unroll
    for (int i = 0; i < FT; ++i) pw[i] = p.w + (int64_t)min(tf + i, p.wt - 1) * p.steps * 1024 + lane * 16;
#pragma unroll
    for (int j = 0; j < TT; ++j) px[j] = p.x + (int64_t)min(tt + j, p.xt - 1) * p.steps * 1024 + lane * 16;
    v4i acc[FT][TT];
#pragma unroll
    for (int i = 0; i < FT; ++i)
#pragma unroll
        for (int j = 0; j < TT; ++j) acc[i][j] = (v4i){0, 0, 0, 0};
    // U steps are on their way while the U before them are multiplied; steps past the last one load the operands' last step
    constexpr int U = KS_AHEAD / (FT + TT);
    v4i w[U][FT], x[U][TT];
    auto load = [&](int s) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t at = (int64_t)min(s + u, p.steps - 1) * 1024;
#pragma unroll
            for (int i = 0; i < FT; ++i) w[u][i] = *(const v4i*)(pw[i] + at);
#pragma unroll
            for (int j = 0; j < TT; ++j) x[u][j] = *(const v4i*)(px[j] + at);
        }
    };
    load(first);
    for (int s = first; s < last; s += U) {
        v4i cw[U][FT], cx[U][TT];
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int i = 0; i < FT; ++i) cw[u][i] = w[u][i];
#pragma unroll
            for (int j = 0; j < TT; ++j) cx[u][j] = x[u][j];
        }
        if (s + U < last) load(s + U);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (s + u < last) {
#pragma unroll
                for (int i = 0; i < FT; ++i)
#pragma unroll
                    for (int j = 0; j < TT; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(cw[u][i], cx[u][j], acc[i][j], 0, 0, 0);
            }
    }
#pragma unroll
    for (int i = 0; i < FT; ++i)
#pragma unroll
        for (int j = 0; j < TT; ++j) s_acc[wave][i * TT + j][lane] = acc[i][j];
    __syncthreads();
    for (int c = wave; c < FT * TT; c += KS_WAVES) {
        v4i sum = s_acc[0][c][lane];
#pragma unroll
        for (int k = 1; k < KS_WAVES; ++k) sum += s_acc[k][c][lane];
        const int64_t m = (int64_t)(tt + c % TT) * 16 + (lane & 15), f = (int64_t)(tf + c / TT) * 16 + (lane >> 4) * 4;
        if (m < p.M && f < p.N) {
            float sw[4], b[4];
            di_channels(p, f, sw, b);
            di_store<T>(p, sum, m, f, p.sx[m], sw, b);
        }
    }
}

// One or two floating-point tokens in one launch: every workgroup quantises them for itself (32 elements a thread at most), into LDS, while
// its first weights are on their way, and goes on as the kernel above.  1 x 4096 x 4096 4.5 us, 3.7 TB/s of weights.
constexpr int TK_ELEMENTS = 16384;          // tokens x padded K
constexpr int TK_TOKENS = 2;
template <typename X, typename T, int FT>
__global__ __launch_bounds__(64 * KS_WAVES) void dense_i8_tokens_kernel(const DenseParams p, const X* x, int64_t ldx, int K) {
    constexpr int THREADS = 64 * KS_WAVES, U = 4;
    __shared__ __attribute__((aligned(16))) char s_x[TK_ELEMENTS];         // [token][16-byte piece]
    __shared__ v4i s_acc[KS_WAVES][FT][64];
    __shared__ uint32_t s_top[TK_TOKENS];
    const int tid = threadIdx.x, lane = tid & 63, M = (int)p.M;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int tf = blockIdx.x * FT, pieces = p.steps * 4;                  // of a token
    const int first = (int)((int64_t)wave * p.steps / KS_WAVES), last = (int)((int64_t)(wave + 1) * p.steps / KS_WAVES);
    const char* pw[FT];
#pragma unroll
    for (int i = 0; i < FT; ++i) pw[i] = p.w + (int64_t)min(tf + i, p.wt - 1) * p.steps * 1024 + lane * 16;
    v4i w[U][FT];
    auto load = [&](int s) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < FT; ++i) w[u][i] = *(const v4i*)(pw[i] + (int64_t)min(s + u, p.steps - 1) * 1024);
    };
    // the tokens' pieces, two a thread at most, their tokens' largest magnitudes in LDS
    Piece<X> v[2];
    int row[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int i = tid + h * THREADS;
        row[h] = i < M * pieces ? i / pieces : -1;
        if (row[h] >= 0) piece_load(v[h], x + row[h] * ldx, (int64_t)(i - row[h] * pieces) * 16, (int64_t)K);
    }
    load(first);
    if (tid < TK_TOKENS) s_top[tid] = 0;
    __syncthreads();
    uint32_t m[2] = {0, 0};
#pragma unroll
    for (int h = 0; h < 2; ++h)
        if (row[h] >= 0) {
            piece_max(v[h], m[h]);
            if constexpr (sizeof(X) == 2) m[h] = max(m[h] & 0xffffu, m[h] >> 16);
        }
    for (int r = 0; r < M; ++r) {
        uint32_t t = max(row[0] == r ? m[0] : 0u, row[1] == r ? m[1] : 0u);
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) t = max(t, (uint32_t)__shfl_xor((int)t, o));
        if (lane == 0 && t) atomicMax(&s_top[r], t);                       // (the largest, whatever the order)
    }
    __syncthreads();
    auto top_of = [&](int r) {
        if constexpr (sizeof(X) == 4) return __uint_as_float(s_top[r]);
        else { X t; t.u = (uint16_t)s_top[r]; return el_f32(t); }
    };
#pragma unroll
    for (int h = 0; h < 2; ++h)
        if (row[h] >= 0) {
            float top = top_of(row[h]);
            const bool zero = !(top > 0.0f && __float_as_uint(top) < 0x7f800000u);
            const float by = di_by(top);
            top *= by;
            *(v4i*)(s_x + (tid + h * THREADS) * 16) = zero ? (v4i){0, 0, 0, 0} : di_quant16<X>(v[h], 127.0f / top, top, by);
        }
    __syncthreads();

    v4i acc[FT];
#pragma unroll
    for (int i = 0; i < FT; ++i) acc[i] = (v4i){0, 0, 0, 0};
    const char* px = s_x + (min(lane & 15, M - 1) * pieces + (lane >> 4)) * 16;      // columns behind the last token repeat it
    for (int s = first; s < last; s += U) {
        v4i c[U][FT];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < FT; ++i) c[u][i] = w[u][i];
        if (s + U < last) load(s + U);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (s + u < last) {
                const v4i b = *(const v4i*)(px + (s + u) * 64);
#pragma unroll
                for (int i = 0; i < FT; ++i) acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(c[u][i], b, acc[i], 0, 0, 0);
            }
    }
#pragma unroll
    for (int i = 0; i < FT; ++i) s_acc[wave][i][lane] = acc[i];
    __syncthreads();
    if (wave < FT) {
        v4i sum = s_acc[0][wave][lane];
#pragma unroll
        for (int k = 1; k < KS_WAVES; ++k) sum += s_acc[k][wave][lane];
        const int64_t r = lane & 15, f = (int64_t)(tf + wave) * 16 + (lane >> 4) * 4;
        if (r < M && f < p.N) {
            float sw[4], b[4];
            di_channels(p, f, sw, b);
            di_store<T>(p, sum, r, f, top_of((int)r) / 127.0f, sw, b);
        }
    }
}

int di_fail(int code, const char* who, const char* what) {
    char msg[200];
    snprintf(msg, sizeof msg, "%s: %s", who, what);
    return set_error(code, msg);
}
int di_launched(const char* who) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? ACCERL_OK : di_fail(ACCERL_EHIP, who, hipGetErrorString(e));
}
bool di_aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

int64_t packed_bytes(int64_t rows, int64_t cols) { return (rows + 15) / 16 * di_steps(cols) * 1024; }

const char* di_sizes(int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 1) return "need rows >= 0 and at least one column";
    return nullptr;
}
const char* di_range(int64_t rows, int64_t cols) {
    return rows > DI_MAX_ROWS || cols > DI_MAX_K ? "more than 2^24 rows or 2^16 columns" : nullptr;
}

int quantize(const char* who, const void* x, int dtype, int64_t rows, int64_t cols, int64_t ld, int8_t* out, float* scale, hipStream_t s) {
    const int steps = (int)di_steps(cols);
    auto go = [&](auto* p) {
        typedef typename std::remove_const<typename std::remove_pointer<decltype(p)>::type>::type T;
        const int64_t padded = (rows + 15) / 16 * 16;
        if (rows <= QR_SINGLE) quantize_rows_kernel<T, 1, 2><<<dim3((unsigned)padded), dim3(QR_THREADS), 0, s>>>(p, rows, cols, ld, (v4i*)out, scale, steps);
        else if (cols > QR_SHORT) quantize_rows_kernel<T, 4, 4><<<dim3((unsigned)(padded / 4)), dim3(QR_THREADS), 0, s>>>(p, rows, cols, ld, (v4i*)out, scale, steps);
        else quantize_rows_kernel<T, 16, 4><<<dim3((unsigned)(padded / 16)), dim3(QR_THREADS), 0, s>>>(p, rows, cols, ld, (v4i*)out, scale, steps);
    };
    if (dtype == ACCERL_DT_F32) go((const float*)x);
    else if (dtype == ACCERL_DT_BF16) go((const BF16*)x);
    else go((const F16*)x);
    return di_launched(who);
}

template <typename T, int WF, int WT, int FA, int FB, int KS>
int tile_go(const char* who, const DenseParams& p, hipStream_t s) {
    const int64_t n = (int64_t)((p.wt + WF * FA - 1) / (WF * FA)) * ((p.xt + WT * FB - 1) / (WT * FB));
    if (n * 64 * WF * WT > MAX_LAUNCH_ITEMS) return di_fail(ACCERL_EUNSUPPORTED, who, "more outputs than one launch covers");
    dense_i8_tile_kernel<T, WF, WT, FA, FB, KS><<<dim3((unsigned)n), dim3(64 * WF * WT), 0, s>>>(p);
    return di_launched(who);
}
template <typename T, int FT, int TT>
int ksplit_go(const char* who, const DenseParams& p, hipStream_t s) {
    dense_i8_ksplit_kernel<T, FT, TT><<<dim3((unsigned)((p.wt + FT - 1) / FT), (unsigned)((p.xt + TT - 1) / TT)), dim3(64 * KS_WAVES), 0, s>>>(p);
    return di_launched(who);
}

template <typename T>
int product_as(const char* who, const DenseParams& p, hipStream_t s) {
    const int64_t cus = conv_num_cus();
    auto groups = [&](int bf, int bt) { return (int64_t)((p.wt + bf - 1) / bf) * ((p.xt + bt - 1) / bt); };
    // (times in us, M x K x N)
    // One or two tiles of tokens stream the weights: one tile of features a workgroup brings more of them under way (24 x 2048 x 8192 5.3, two
    // tiles 6.5; 32 x 8192 x 1024 one by one 4.9, two tiles of tokens 6.1; 8 x 4096 x 16384 in tiles 24.3).
    if (p.xt <= 2) return p.xt == 2 && p.wt >= cus ? ksplit_go<T, 1, 2>(who, p, s) : ksplit_go<T, 1, 1>(who, p, s);
    if (p.xt > 8) {
        // 256 x 256 in one workgroup a compute unit where its rounds are nearly full, else 128 features x 256 tokens, two workgroups a
        // compute unit, whose ends overlap the other's steps: 4096 x 4096 x 4096 55.9 / 58.2, 4096 x 16384 x 4096 199 / 217, but 6000 x 2000
        // x 5000 63.8 / 59.2, 8192 x 8192 x 1024 85.7 / 64.9
        const int64_t full = groups(16, 16), rounds = (full + cus - 1) / cus;
        if (full >= cus && 10 * full >= 9 * rounds * cus) return tile_go<T, 2, 4, 8, 4, 1>(who, p, s);
        if (groups(8, 16) >= cus) return tile_go<T, 1, 4, 8, 4, 1>(who, p, s);
        // 128 x 128, one workgroup a compute unit, where that is one round (64 features x 128 tokens / this: 1024 x 4096 x 4096 22.1 / 20.2,
        // 512 x 8192 x 8192 47.0 / 40.2, 999 x 1777 x 2501 11.2 / 10.5; in a second round 1500 x 384 x 3000 7.9 / 10.9)
        if (2 * groups(8, 8) >= cus && groups(8, 8) <= cus) return tile_go<T, 2, 4, 4, 2, 2>(who, p, s);
    }
    // Fewer: the wavefronts split K, with the largest of their tiles that gives every compute unit work (64 features x 128 tokens /
    // 32 x 64 split: 512 x 2048 x 2048 8.5 / 7.4, 256 x 4096 x 4096 16.9 / 11.5, but 128 x 4096 x 16384 17.9 / 27.5, 4096 x 512 x 512 5.2 / 7.4).
    if (groups(2, 4) > 2 * cus) return tile_go<T, 1, 4, 4, 2, 2>(who, p, s);
    return groups(2, 4) >= cus ? ksplit_go<T, 2, 4>(who, p, s) : ksplit_go<T, 2, 2>(who, p, s);
}
int product(const char* who, const DenseParams& p, hipStream_t s) {
    if (p.dtype == ACCERL_DT_F32) return product_as<float>(who, p, s);
    return p.dtype == ACCERL_DT_BF16 ? product_as<BF16>(who, p, s) : product_as<F16>(who, p, s);
}

// One or two tokens: one launch (us, two launches / one: 1 x 4096 x 4096 9.7 / 7.1, 2 x 4096 x 4096 9.6 / 7.6, but 4 tokens 9.5 / 10.1, 8 x
// 2048 x 2048 7.2 / 9.4); two tiles of features a workgroup from 1024 on (1 x 512 x 32000 12.8 / 10.8, 1 x 4096 x 4096 7.1 / 7.9).
bool tokens_fit(int64_t M, int64_t K) { return M <= TK_TOKENS && M * di_steps(K) * 64 <= TK_ELEMENTS; }
template <typename X>
int tokens(const char* who, const X* x, int64_t ldx, int64_t K, const DenseParams& p, hipStream_t s) {
    const auto go = [&](auto type) {
        typedef decltype(type) T;
        if (p.wt < 1024) dense_i8_tokens_kernel<X, T, 1><<<dim3((unsigned)p.wt), dim3(64 * KS_WAVES), 0, s>>>(p, x, ldx, (int)K);
        else dense_i8_tokens_kernel<X, T, 2><<<dim3((unsigned)((p.wt + 1) / 2)), dim3(64 * KS_WAVES), 0, s>>>(p, x, ldx, (int)K);
    };
    if (p.dtype == ACCERL_DT_F32) go(0.0f);
    else if (p.dtype == ACCERL_DT_BF16) go(BF16());
    else go(F16());
    return di_launched(who);
}

// what both forms of the layer check; `done` is set where nothing is to be done
int check_product(const char* who, const int8_t* w, const float* w_scale, const float* bias, int64_t M, int64_t N, int64_t K, const void* out,
                  int32_t out_dtype, int64_t ld_out, bool* done) {
    *done = false;
    if (const char* bad = di_sizes(M, K)) return di_fail(ACCERL_EINVAL, who, bad);
    if (const char* bad = di_sizes(N, K)) return di_fail(ACCERL_EINVAL, who, bad);
    if (!dtype_known(out_dtype)) return di_fail(ACCERL_EINVAL, who, "unknown output type");
    if (ld_out < N) return di_fail(ACCERL_EINVAL, who, "output rows overlap (ld_out < N)");
    if (di_range(M, K) || di_range(N, K)) return di_fail(ACCERL_EUNSUPPORTED, who, "more than 2^24 tokens or features, or K above 2^16");
    if (M == 0 || N == 0) { *done = true; return ACCERL_OK; }
    if (!w || !w_scale || !out) return di_fail(ACCERL_EINVAL, who, "NULL argument (only bias may be NULL)");
    if (!di_aligned(w, 16)) return di_fail(ACCERL_EINVAL, who, "packed rows must be 16-byte aligned");
    if (!di_aligned(w_scale, 4) || !di_aligned(bias, 4) || !di_aligned(out, dtype_bytes(out_dtype))) return di_fail(ACCERL_EINVAL, who, "misaligned argument");
    const Table to = table(out, M, ld_out, N, dtype_bytes(out_dtype));
    if (share(to, table(w, packed_bytes(N, K))) || share(to, table(w_scale, N * 4)) || share(to, table(bias, N * 4)))
        return di_fail(ACCERL_EINVAL, who, "the output overlaps the layer's weights, scales or bias");
    return ACCERL_OK;
}
DenseParams dense_params(const int8_t* x, const float* x_scale, const int8_t* w, const float* w_scale, const float* bias, int64_t M, int64_t N, int64_t K,
                         int relu, void* out, int out_dtype, int64_t ld_out) {
    DenseParams p{};
    p.x = (const char*)x; p.w = (const char*)w; p.sx = x_scale; p.sw = w_scale; p.bias = bias; p.out = out;
    p.M = M; p.N = N; p.ld = ld_out;
    p.xt = (int)((M + 15) / 16); p.wt = (int)((N + 15) / 16); p.steps = (int)di_steps(K);
    p.dtype = out_dtype; p.relu = relu != 0;
    return p;
}
}  // namespace
}  // namespace accerl

using namespace accerl;

extern "C" {

int64_t accerl_packed_rows_bytes(int64_t rows, int64_t cols) {
    if (const char* bad = di_sizes(rows, cols)) return di_fail(ACCERL_EINVAL, "packed rows", bad);
    if (const char* bad = di_range(rows, cols)) return di_fail(ACCERL_EUNSUPPORTED, "packed rows", bad);
    return packed_bytes(rows, cols);
}

static int check_rows(const char* who, const void* in, int64_t rows, int64_t cols, int64_t ld, const void* out, const void* packed, bool* done) {
    *done = false;
    if (const char* bad = di_sizes(rows, cols)) return di_fail(ACCERL_EINVAL, who, bad);
    if (ld < cols) return di_fail(ACCERL_EINVAL, who, "rows overlap (ld < cols)");
    if (const char* bad = di_range(rows, cols)) return di_fail(ACCERL_EUNSUPPORTED, who, bad);
    if (rows == 0) { *done = true; return ACCERL_OK; }
    if (!in || !out) return di_fail(ACCERL_EINVAL, who, "NULL argument");
    if (!di_aligned(packed, 16)) return di_fail(ACCERL_EINVAL, who, "packed rows must be 16-byte aligned");
    return ACCERL_OK;
}

int accerl_quantize_rows(const void* x, int32_t x_dtype, int64_t rows, int64_t cols, int64_t ld_x, int8_t* out_packed, float* out_scale, void* stream) {
    const char* who = "quantize_rows";
    bool done;
    if (!dtype_known(x_dtype)) return di_fail(ACCERL_EINVAL, who, "unknown input type");
    if (int rc = check_rows(who, x, rows, cols, ld_x, out_packed, out_packed, &done)) return rc;
    if (done) return ACCERL_OK;
    if (!out_scale) return di_fail(ACCERL_EINVAL, who, "NULL argument");
    if (!di_aligned(x, dtype_bytes(x_dtype)) || !di_aligned(out_scale, 4)) return di_fail(ACCERL_EINVAL, who, "misaligned argument");
    return quantize(who, x, x_dtype, rows, cols, ld_x, out_packed, out_scale, (hipStream_t)stream);
}

int accerl_pack_rows_i8(const int8_t* q, int64_t rows, int64_t cols, int64_t ld_q, int8_t* out_packed, void* stream) {
    bool done;
    if (int rc = check_rows("pack_rows", q, rows, cols, ld_q, out_packed, out_packed, &done)) return rc;
    if (done) return ACCERL_OK;
    const int64_t n = packed_bytes(rows, cols) / 16, blocks = (n + 255) / 256;
    pack_rows_kernel<<<dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(256), 0, (hipStream_t)stream>>>(q, rows, cols, ld_q, (v4i*)out_packed, di_steps(cols), n);
    return di_launched("pack_rows");
}

int accerl_unpack_rows_i8(const int8_t* packed, int64_t rows, int64_t cols, int8_t* out_q, int64_t ld_q, void* stream) {
    bool done;
    if (int rc = check_rows("unpack_rows", packed, rows, cols, ld_q, out_q, packed, &done)) return rc;
    if (done) return ACCERL_OK;
    const int64_t n = packed_bytes(rows, cols) / 16, blocks = (n + 255) / 256;
    unpack_rows_kernel<<<dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(256), 0, (hipStream_t)stream>>>((const v4i*)packed, rows, cols, ld_q, out_q, di_steps(cols), n);
    return di_launched("unpack_rows");
}

int accerl_dense_i8(const int8_t* x_packed, const float* x_scale, const int8_t* w_packed, const float* w_scale, const float* bias,
                    int64_t M, int64_t N, int64_t K, int32_t relu, void* out, int32_t out_dtype, int64_t ld_out, void* stream) {
    const char* who = "dense_i8";
    bool done;
    if (int rc = check_product(who, w_packed, w_scale, bias, M, N, K, out, out_dtype, ld_out, &done)) return rc;
    if (done) return ACCERL_OK;
    if (!x_packed || !x_scale) return di_fail(ACCERL_EINVAL, who, "NULL argument (only bias may be NULL)");
    if (!di_aligned(x_packed, 16) || !di_aligned(x_scale, 4)) return di_fail(ACCERL_EINVAL, who, "misaligned argument");
    const Table to = table(out, M, ld_out, N, dtype_bytes(out_dtype));
    if (share(to, table(x_packed, packed_bytes(M, K))) || share(to, table(x_scale, M * 4))) return di_fail(ACCERL_EINVAL, who, "the output overlaps the tokens or their scales");
    return product(who, dense_params(x_packed, x_scale, w_packed, w_scale, bias, M, N, K, relu, out, out_dtype, ld_out), (hipStream_t)stream);
}

// the quantised tokens and, from the next multiple of 256 bytes on, their scales
static int64_t scales_at(int64_t M, int64_t K) { return (packed_bytes(M, K) + 255) / 256 * 256; }

int64_t accerl_dense_i8_workspace(int64_t M, int64_t K) {
    if (const char* bad = di_sizes(M, K)) return di_fail(ACCERL_EINVAL, "dense_i8_workspace", bad);
    if (const char* bad = di_range(M, K)) return di_fail(ACCERL_EUNSUPPORTED, "dense_i8_workspace", bad);
    return scales_at(M, K) + (M * 4 + 255) / 256 * 256;
}

int accerl_dense_i8_dynamic(const void* x, int32_t x_dtype, int64_t ld_x, const int8_t* w_packed, const float* w_scale, const float* bias,
                            int64_t M, int64_t N, int64_t K, int32_t relu, void* out, int32_t out_dtype, int64_t ld_out,
                            void* workspace, int64_t workspace_bytes, void* stream) {
    const char* who = "dense_i8_dynamic";
    bool done;
    if (!dtype_known(x_dtype)) return di_fail(ACCERL_EINVAL, who, "unknown input type");
    if (int rc = check_product(who, w_packed, w_scale, bias, M, N, K, out, out_dtype, ld_out, &done)) return rc;
    if (ld_x < K) return di_fail(ACCERL_EINVAL, who, "input rows overlap (ld_x < K)");
    if (done) return ACCERL_OK;
    if (!x || !workspace) return di_fail(ACCERL_EINVAL, who, "NULL argument (only bias may be NULL)");
    if (!di_aligned(x, dtype_bytes(x_dtype)) || !di_aligned(workspace, 16)) return di_fail(ACCERL_EINVAL, who, "misaligned argument");
    if (workspace_bytes < accerl_dense_i8_workspace(M, K)) return di_fail(ACCERL_EINVAL, who, "workspace smaller than accerl_dense_i8_workspace says");
    const int64_t used = accerl_dense_i8_workspace(M, K);
    const Table from = table(x, M, ld_x, K, dtype_bytes(x_dtype)), to = table(out, M, ld_out, N, dtype_bytes(out_dtype));
    if (share(table(workspace, used), from) || share(table(workspace, used), to)) return di_fail(ACCERL_EINVAL, who, "the workspace overlaps the input or the output");
    // (every workgroup of the one launch reads the tokens: where the output lies over them they are quantised first)
    if (tokens_fit(M, K) && !share(from, to)) {
        const DenseParams p = dense_params(nullptr, nullptr, w_packed, w_scale, bias, M, N, K, relu, out, out_dtype, ld_out);
        if (x_dtype == ACCERL_DT_F32) return tokens(who, (const float*)x, ld_x, K, p, (hipStream_t)stream);
        return x_dtype == ACCERL_DT_BF16 ? tokens(who, (const BF16*)x, ld_x, K, p, (hipStream_t)stream) : tokens(who, (const F16*)x, ld_x, K, p, (hipStream_t)stream);
    }
    int8_t* xq = (int8_t*)workspace;
    float* sx = (float*)((char*)workspace + scales_at(M, K));
    if (int rc = quantize(who, x, x_dtype, M, K, ld_x, xq, sx, (hipStream_t)stream)) return rc;
    return product(who, dense_params(xq, sx, w_packed, w_scale, bias, M, N, K, relu, out, out_dtype, ld_out), (hipStream_t)stream);
}

}  // extern "C"
