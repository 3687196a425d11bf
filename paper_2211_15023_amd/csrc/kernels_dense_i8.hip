// Int8 dense layers whose inputs are quantised with a scale for each token (row) and whose weights have one for each channel:
//   s_x[m] = max_k |x[m,k]| / 127,  q[m,k] = rint(x[m,k] * 127 / max),  y[m,n] = (sum_k q[m,k] w[n,k]) s_x[m] s_w[n] + b[n].
//
// Both operands lie packed in the order in which the matrix instruction takes them: tiles of 16 rows x 64 bytes of K,
// [row tile][k step][lane = 16 * (k % 64 / 16) + row % 16][16 bytes], K padded with zeros to whole pairs of steps.  A tile is one
// contiguous KiB, so every operand load is one coalesced access, goes to LDS without passing registers, and is read back from there
// without bank conflicts; no kernel meets a K that ends inside a step.  Features are the matrix instruction's rows: a lane ends up
// with four consecutive features of one token.
#include <stdio.h>

#include "wide_ops.h"

namespace accerl {

int conv_num_cus();   // compute units of the current device

namespace {

constexpr int64_t DI_MAX_ROWS = 1 << 24, DI_MAX_K = 1 << 16;      // 2^16 * 128 * 128 is half of what an int32 sum holds

__host__ __device__ inline int64_t di_steps(int64_t K) { return (K + 127) / 128 * 2; }

// ---------------------------------------------------------------- quantising
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

// sixteen elements of a row from element k on; what lies past the row's end is zero
template <typename T>
__device__ __forceinline__ void di_load16(const T* row, int64_t k, int64_t cols, float (&v)[16]) {
    if (k + 16 <= cols) {
        if constexpr (__is_same(T, float)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                typedef u32x4 u32x4_at4 __attribute__((aligned(4)));
                const u32x4 w = *(const u32x4_at4*)(row + k + 4 * i);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[4 * i + e] = __uint_as_float(w[e]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const u32x4 w = *(const u32x4_at2*)(row + k + 8 * i);
#pragma unroll
                for (int e = 0; e < 4; ++e) el_pair<T>(w[e], v[8 * i + 2 * e], v[8 * i + 2 * e + 1]);
            }
        }
    } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = k + e < cols ? el_f32(row[k + e]) : 0.0f;
    }
}

// A workgroup quantises 16 rows, one row tile: lane l of a wavefront is row l % 16 and one of four pieces of 16 elements, so that a
// wavefront reads 16 rows' runs of 64 elements and writes a whole KiB.  Magnitudes are compared as integers, in which a NaN is larger
// than everything: a row that holds a NaN or an infinity gets it as its scale and zeros, so that its results are NaN.
constexpr int QR_THREADS = 1024;
template <typename T>
__global__ __launch_bounds__(QR_THREADS) void quantize_rows_kernel(const T* x, int64_t rows, int64_t cols, int64_t ld, v4i* out, float* scale, int steps) {
    __shared__ uint32_t s_max[QR_THREADS / 64][16];
    const int tid = threadIdx.x, r = tid & 15, piece = tid >> 4;
    const int64_t row = (int64_t)blockIdx.x * 16 + r;
    const bool real = row < rows;
    const T* src = x + (real ? row : rows - 1) * ld;
    float v[16];
    uint32_t m = 0;
    for (int64_t k = piece * 16; k < cols; k += QR_THREADS) {
        di_load16(src, k, cols, v);
#pragma unroll
        for (int e = 0; e < 16; ++e) m = max(m, __float_as_uint(v[e]) & 0x7fffffffu);
    }
    m = max(m, (uint32_t)__shfl_xor((int)m, 16));
    m = max(m, (uint32_t)__shfl_xor((int)m, 32));
    if ((tid & 63) < 16) s_max[tid >> 6][r] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < QR_THREADS / 64; ++w) m = max(m, s_max[w][r]);
    float top = __uint_as_float(m);
    if (real && piece == 0) scale[row] = top / 127.0f;
    // scaled by a power of two where 127 / max or 127 * x would leave the range
    float by = top < 0x1p-100f ? 0x1p100f : top > 0x1p100f ? 0x1p-20f : 1.0f;
    const bool zero = !real || !(top > 0.0f && m < 0x7f800000u);
    top *= by;
    const float inv = 127.0f / top;
    v4i* dst = out + (int64_t)blockIdx.x * steps * 64 + r;
    for (int p = piece; p < steps * 4; p += QR_THREADS / 16) {
        v4i o = {0, 0, 0, 0};
        if (!zero && (int64_t)p * 16 < cols) {
            di_load16(src, (int64_t)p * 16, cols, v);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                uint32_t u = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) u |= ((uint32_t)di_quant<T>(v[4 * w + e] * by, inv, top) & 0xffu) << (8 * e);
                o[w] = (int)u;
            }
        }
        dst[p * 16] = o;
    }
}

// int8 rows to tiles and back, a 16-byte piece a thread
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

// results of features n .. n + 3 of token m
template <typename T>
__device__ __forceinline__ void di_store(const DenseParams& p, const v4i& acc, int64_t m, int64_t n, float sx, const float (&sw)[4], const float (&b)[4]) {
    float y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        y[e] = fmaf((float)acc[e] * sx, sw[e], b[e]);
        if (p.relu) y[e] = y[e] < 0.0f ? 0.0f : y[e];             // a NaN stays
    }
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

#define DI_GLOBAL(q) ((const __attribute__((address_space(1))) void*)(q))
#define DI_LDS(q) ((__attribute__((address_space(3))) void*)(q))

// Large products.  A workgroup of WF x WT wavefronts owns (16 WF FA) features x (16 WT FB) tokens and walks K in stages of two steps
// (128 bytes of every row).  A stage's fragments go to one of two LDS buffers while the other is multiplied from; two arrays
// and pointers that do not alias let the compiler keep a stage's loads in flight across the reads of the other buffer.
template <int FA, int FB>
struct Frags { v4i a[FA], b[FB]; };

template <int WF, int WT, int FA, int FB>
__device__ __forceinline__ void di_fetch(char* __restrict__ dst, const char* const (&src)[(WF * FA + WT * FB) * 2 / (WF * WT)], int64_t at, int wave) {
    constexpr int PER = (WF * FA + WT * FB) * 2 / (WF * WT);
#pragma unroll
    for (int i = 0; i < PER; ++i)
        __builtin_amdgcn_global_load_lds(DI_GLOBAL(src[i] + at), DI_LDS(dst + (wave * PER + i) * 1024), 16, 0, 0);
}

template <int WF, int WT, int FA, int FB>
__device__ __forceinline__ void di_stage(const char* __restrict__ cur, char* __restrict__ nxt, const char* const (&src)[(WF * FA + WT * FB) * 2 / (WF * WT)],
                                         int64_t at, bool more, int wave, int wf, int wt, int lane, v4i (&acc)[FA][FB]) {
    if (more) di_fetch<WF, WT, FA, FB>(nxt, src, at, wave);
    const char* pa = cur + wf * FA * 2048 + lane * 16;
    const char* pb = cur + (WF * FA + wt * FB) * 2048 + lane * 16;
#pragma unroll
    for (int st = 0; st < 2; ++st) {
        Frags<FA, FB> f;
#pragma unroll
        for (int i = 0; i < FB; ++i) f.b[i] = *(const v4i*)(pb + (2 * i + st) * 1024);
#pragma unroll
        for (int i = 0; i < FA; ++i) f.a[i] = *(const v4i*)(pa + (2 * i + st) * 1024);
#pragma unroll
        for (int i = 0; i < FA; ++i)
#pragma unroll
            for (int j = 0; j < FB; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(f.a[i], f.b[j], acc[i][j], 0, 0, 0);
    }
}

template <typename T, int WF, int WT, int FA, int FB>
__global__ __launch_bounds__(64 * WF * WT) void dense_i8_tile_kernel(const DenseParams p) {
    constexpr int BF = WF * FA, BT = WT * FB;                       // row tiles of a workgroup
    constexpr int STAGE = (BF + BT) * 2048;
    constexpr int PER = (BF + BT) * 2 / (WF * WT);                  // fragments a wavefront fetches per stage
    static_assert((BF + BT) * 2 % (WF * WT) == 0, "whole fragments a wavefront");
    __shared__ __attribute__((aligned(16))) char s0[STAGE];
    __shared__ __attribute__((aligned(16))) char s1[STAGE];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wf = wave % WF, wt = wave / WF;

    // Workgroup n runs on XCD n mod 8.  Every XCD takes consecutive tiles of an order that walks squares of up to 4 x 8 tiles, so
    // that the workgroups that run together on it share rows in its cache.
    const unsigned gf = (p.wt + BF - 1) / BF, gt = (p.xt + BT - 1) / BT, n = gf * gt, id = blockIdx.x, xcd = id & 7;
    const unsigned t = xcd * (n >> 3) + min(xcd, n & 7) + (id >> 3);
    constexpr unsigned GROUP = 4;
    const unsigned band = t / (GROUP * gf), first = band * GROUP, high = min(GROUP, gt - first), in = t - band * GROUP * gf;
    const int tf = (int)(in / high) * BF, tt = (int)(first + in % high) * BT;

    // a tile past the end re-reads the last one; its results are not stored
    const char* src[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int f = wave * PER + i, tile = f >> 1, st = f & 1;
        src[i] = tile < BF ? p.w + ((int64_t)min(tf + tile, p.wt - 1) * p.steps + st) * 1024
                           : p.x + ((int64_t)min(tt + tile - BF, p.xt - 1) * p.steps + st) * 1024;
        src[i] += lane * 16;
    }
    v4i acc[FA][FB];
#pragma unroll
    for (int i = 0; i < FA; ++i)
#pragma unroll
        for (int j = 0; j < FB; ++j) acc[i][j] = (v4i){0, 0, 0, 0};

    const int stages = p.steps >> 1;
    di_fetch<WF, WT, FA, FB>(s0, src, 0, wave);
    __syncthreads();
    int s = 0;
    for (; s + 2 <= stages; s += 2) {
        di_stage<WF, WT, FA, FB>(s0, s1, src, (int64_t)(s + 1) * 2048, true, wave, wf, wt, lane, acc);
        __syncthreads();
        di_stage<WF, WT, FA, FB>(s1, s0, src, (int64_t)(s + 2) * 2048, s + 2 < stages, wave, wf, wt, lane, acc);
        __syncthreads();
    }
    if (s < stages) di_stage<WF, WT, FA, FB>(s0, s1, src, 0, false, wave, wf, wt, lane, acc);

    float sx[FB];
    int64_t m[FB];
#pragma unroll
    for (int j = 0; j < FB; ++j) {
        m[j] = (int64_t)(tt + wt * FB + j) * 16 + (lane & 15);
        sx[j] = p.sx[min(m[j], p.M - 1)];
    }
#pragma unroll
    for (int i = 0; i < FA; ++i) {
        const int64_t f = (int64_t)(tf + wf * FA + i) * 16 + (lane >> 4) * 4;
        float sw[4], b[4];
        di_channels(p, f, sw, b);
#pragma unroll
        for (int j = 0; j < FB; ++j)
            if (m[j] < p.M && f < p.N) di_store<T>(p, acc[i][j], m[j], f, sx[j], sw, b);
    }
}

// Few tokens or few tiles: the eight wavefronts of a workgroup split K, each multiplies straight from memory (a weight is read once, by
// one wavefront), and their sums meet in LDS.
constexpr int KS_WAVES = 8;
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
    constexpr int U = 4;
    int s = first;
    for (; s + U <= last; s += U) {
        v4i w[U][FT], x[U][TT];
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int i = 0; i < FT; ++i) w[u][i] = *(const v4i*)(pw[i] + (int64_t)(s + u) * 1024);
#pragma unroll
            for (int j = 0; j < TT; ++j) x[u][j] = *(const v4i*)(px[j] + (int64_t)(s + u) * 1024);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < FT; ++i)
#pragma unroll
                for (int j = 0; j < TT; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[u][i], x[u][j], acc[i][j], 0, 0, 0);
    }
    for (; s < last; ++s) {
        v4i w[FT], x[TT];
#pragma unroll
        for (int i = 0; i < FT; ++i) w[i] = *(const v4i*)(pw[i] + (int64_t)s * 1024);
#pragma unroll
        for (int j = 0; j < TT; ++j) x[j] = *(const v4i*)(px[j] + (int64_t)s * 1024);
#pragma unroll
        for (int i = 0; i < FT; ++i)
#pragma unroll
            for (int j = 0; j < TT; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[i], x[j], acc[i][j], 0, 0, 0);
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

const char* di_sizes(int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 1) return "need rows >= 0 and at least one column";
    return nullptr;
}
const char* di_range(int64_t rows, int64_t cols) {
    return rows > DI_MAX_ROWS || cols > DI_MAX_K ? "more than 2^24 rows or 2^16 columns" : nullptr;
}

int quantize(const char* who, const void* x, int dtype, int64_t rows, int64_t cols, int64_t ld, int8_t* out, float* scale, hipStream_t s) {
    const int steps = (int)di_steps(cols);
    const dim3 grid((unsigned)((rows + 15) / 16)), block(QR_THREADS);
    if (dtype == ACCERL_DT_F32) quantize_rows_kernel<float><<<grid, block, 0, s>>>((const float*)x, rows, cols, ld, (v4i*)out, scale, steps);
    else if (dtype == ACCERL_DT_BF16) quantize_rows_kernel<BF16><<<grid, block, 0, s>>>((const BF16*)x, rows, cols, ld, (v4i*)out, scale, steps);
    else quantize_rows_kernel<F16><<<grid, block, 0, s>>>((const F16*)x, rows, cols, ld, (v4i*)out, scale, steps);
    return di_launched(who);
}

template <typename T, int WF, int WT, int FA, int FB>
int tile_go(const char* who, const DenseParams& p, hipStream_t s) {
    const int64_t n = (int64_t)((p.wt + WF * FA - 1) / (WF * FA)) * ((p.xt + WT * FB - 1) / (WT * FB));
    if (n * 64 * WF * WT > MAX_LAUNCH_ITEMS) return di_fail(ACCERL_EUNSUPPORTED, who, "more outputs than one launch covers");
    dense_i8_tile_kernel<T, WF, WT, FA, FB><<<dim3((unsigned)n), dim3(64 * WF * WT), 0, s>>>(p);
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
    if (groups(16, 16) >= cus) return tile_go<T, 2, 4, 8, 4>(who, p, s);
    if (groups(8, 8) >= cus) return tile_go<T, 2, 2, 4, 4>(who, p, s);
    if (p.xt == 1) return ksplit_go<T, 1, 1>(who, p, s);
    if (p.xt == 2) return groups(2, 2) >= cus ? ksplit_go<T, 2, 2>(who, p, s) : ksplit_go<T, 1, 2>(who, p, s);
    if (groups(4, 4) >= 2 * cus) return tile_go<T, 2, 2, 2, 2>(who, p, s);
    if (groups(2, 4) >= cus) return ksplit_go<T, 2, 4>(who, p, s);
    return ksplit_go<T, 1, 2>(who, p, s);
}
int product(const char* who, const DenseParams& p, hipStream_t s) {
    if (p.dtype == ACCERL_DT_F32) return product_as<float>(who, p, s);
    return p.dtype == ACCERL_DT_BF16 ? product_as<BF16>(who, p, s) : product_as<F16>(who, p, s);
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
int64_t packed_bytes(int64_t rows, int64_t cols) { return (rows + 15) / 16 * di_steps(cols) * 1024; }
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
    int8_t* xq = (int8_t*)workspace;
    float* sx = (float*)((char*)workspace + scales_at(M, K));
    if (int rc = quantize(who, x, x_dtype, M, K, ld_x, xq, sx, (hipStream_t)stream)) return rc;
    return product(who, dense_params(xq, sx, w_packed, w_scale, bias, M, N, K, relu, out, out_dtype, ld_out), (hipStream_t)stream);
}

}  // extern "C"
