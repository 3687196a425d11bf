// The norms around a block with its gate and its residual, and their gradients.
//
// A row is read once and stays in the registers of its lanes, eight neighbouring elements at a time: all statistics are taken from there, the mean first and then
// the squares around it.  Bound by memory where the row's eights fill its lanes: 65536 x 2048 bf16 with an fp32 stream 376 us (5.0 TB/s; a large copy reaches
// 4.9), gradients of 32768 x 4096 bf16 463 (4.6; two sums over the row in each direction lie between a row's loads and its stores).  Rows of up to 1024 elements
// (gradients and few rows: 512) belong to a part of a wavefront or to a whole one, longer rows to a workgroup.
#include <algorithm>
#include <cfloat>
#include <cstdio>

#include "wide_ops.h"

namespace accerl {
namespace {

constexpr int BN_MAX_D = 16384;

struct NormParams {
    const void *y, *x, *gate, *gu, *gh;
    void *u, *h, *dy, *dx, *dg;
    int64_t ldy, ldx, ldg, ldgu, ldgh, ldu, ldh, lddy, lddx, lddg;
    const float *after, *before;
    float *da, *db;                       // partial sums of the weights' gradients, [record][D of a group]
    int64_t rows;                         // rows x groups
    int64_t step;                         // from a slot's row to its next: a multiple of the groups, so that a slot keeps its weights
    int D, groups, lanes;                 // of a group's row; lanes a row has
    int layer, gate_kind;
    float eps, skip, branch, inv_d;
};

// Eight elements of a row as they lie in memory, and as numbers.  TINY: rows of less than eight, of which `left` are there (the others 0).
template <typename T> struct Eight { u32x4 w[sizeof(T) / 2]; };
template <bool TINY, typename T> __device__ __forceinline__ void load8(const T* p, int left, Eight<T>& o) {
    if constexpr (TINY) {
        T e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = j < left ? p[j] : T{};
        __builtin_memcpy(&o, e, sizeof o);
    } else if constexpr (sizeof(T) == 4) {
        o.w[0] = *(const u32x4_at4*)p;
        o.w[1] = *(const u32x4_at4*)(p + 4);
    } else {
        o.w[0] = *(const u32x4_at2*)p;
    }
}
template <typename T> __device__ __forceinline__ void numbers8(const Eight<T>& v, float* o) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (sizeof(T) == 4) { o[j] = __uint_as_float(v.w[0][j]); o[4 + j] = __uint_as_float(v.w[1][j]); }
        else el_pair<T>(v.w[0][j], o[2 * j], o[2 * j + 1]);
    }
}
// elements from .. to - 1 of eight
template <typename T> __device__ __forceinline__ void store8(T* p, int from, int to, const float* v) {
    if (to - from == 8) {
        if constexpr (sizeof(T) == 4) {
            *(u32x4_at4*)p = __builtin_bit_cast(u32x4, v4f{v[0], v[1], v[2], v[3]});
            *(u32x4_at4*)(p + 4) = __builtin_bit_cast(u32x4, v4f{v[4], v[5], v[6], v[7]});
        } else {
            u32x4 w;
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = f32_pair<T>(v[2 * j], v[2 * j + 1]);
            *(u32x4_at2*)p = w;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) if (j >= from && j < to) p[j] = f32_el<T>(v[j]);
    }
}

// Sums over the lanes of a row: a power of two of neighbours in a wavefront, or the workgroup (at most 16 wavefronts; two buffers in turn, so that one
// barrier is enough).
template <bool GROUP> struct RowSum {
    float (*red)[16][2];
    int lanes, turn = 0;
    __device__ __forceinline__ void operator()(float& a, float& b) {
        if constexpr (GROUP) {
#pragma unroll
            for (int o = 32; o; o >>= 1) { a += __shfl_xor(a, o); b += __shfl_xor(b, o); }
            const int w = threadIdx.x >> 6, n = blockDim.x >> 6;
            if ((threadIdx.x & 63) == 0) { red[turn][w][0] = a; red[turn][w][1] = b; }
            __syncthreads();
            a = b = 0.0f;
            for (int i = 0; i < n; ++i) { a += red[turn][i][0]; b += red[turn][i][1]; }
            turn ^= 1;
        } else {
            for (int o = lanes >> 1; o; o >>= 1) { a += __shfl_xor(a, o); b += __shfl_xor(b, o); }
        }
    }
    __device__ __forceinline__ float operator()(float a) { float b = 0.0f; (*this)(a, b); return a; }
};

// (the reciprocal instruction is off by one in the last place, and the exponential by about (1 + |x|) 2^-24 of itself, as its argument is multiplied by log2 e in fp32; what
// the slopes take of 1 - sigmoid has the last places of 1)
__device__ __forceinline__ float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.0f + __expf(-x)); }

// z -> (z - mean) and the reciprocal root; elements that are not the lane's stay 0
template <int N, bool GROUP, typename Mine> __device__ __forceinline__ float normed(const NormParams& p, RowSum<GROUP>& sum, float* z, const Mine& mine) {
    if (p.layer) {
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) s += z[i];
        const float mean = sum(s) * p.inv_d;
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = mine(i, z[i] - mean);
    }
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) s += z[i] * z[i];
    const float r = 1.0f / sqrtf(sum(s) * p.inv_d + p.eps);
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] *= r;
    return r;
}
// the gradient t by a norm's result (weight taken in) -> by its input, of the normed z and its reciprocal root
template <int N, bool GROUP> __device__ __forceinline__ void through(const NormParams& p, RowSum<GROUP>& sum, float* t, const float* z, float r) {
    float a = 0.0f, b = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) { a += t[i] * z[i]; b += t[i]; }
    sum(a, b);
    a *= p.inv_d;
    b = p.layer ? b * p.inv_d : 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) t[i] = r * (t[i] - b - z[i] * a);
}

// What a row reads, as it lies in memory.
template <typename T, typename S, int NC> struct NormRow { Eight<T> y[NC], gate[NC], gh[NC]; Eight<S> x[NC], gu[NC]; };

// MOST: threads of a workgroup at most.  While a row is worked on the next one's loads are under way, where registers allow it (AHEAD).
template <typename T, typename S, int NC, int MOST, bool GROUP, bool GRAD, bool TINY>
__global__ __launch_bounds__(MOST, MOST == 1024 ? 4 : MOST == 512 || NC == 2 ? 2 : 3) void block_norm_kernel(const NormParams p) {
    constexpr int N = 8 * NC;
    constexpr bool AHEAD = NC <= 2 && MOST <= 512 && sizeof(NormRow<T, S, NC>) <= 160;
    __shared__ float red[GROUP ? 2 : 1][16][2];
    // The widest rows: the weights' sums are in LDS, and the weights come from the caches for every row
    constexpr bool LEAN = GRAD && NC == 4;
    __shared__ float sums[LEAN ? 2 * MOST * N : GRAD && !GROUP ? 256 * N : 1];
    RowSum<GROUP> sum{red, p.lanes};
    const int lane = GROUP ? threadIdx.x : threadIdx.x & (p.lanes - 1);
    const int64_t slot = GROUP ? blockIdx.x : (int64_t)blockIdx.x * (256 / p.lanes) + threadIdx.x / p.lanes;
    const int part = (int)(slot % p.groups), off = part * p.D;
    // A lane's eights begin at `at`.  The row's last one ends with the row and so begins inside the one before, whose elements it reads too but leaves alone
    // (they count as zeros in everything, so that an infinity there is no NaN here):
    // its own are those from `from` to `to` - 1 (none where the row has no eight for the lane, which reads the first).
    int at[NC], from[NC], to[NC];
    bool whole = true;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int k = (c * p.lanes + lane) * 8, in = min(max(p.D - k, 0), 8);
        at[c] = in == 0 ? 0 : TINY ? k : min(k, p.D - 8);
        from[c] = TINY ? 0 : 8 - in;
        to[c] = TINY ? in : 8;
    }
    whole = !TINY && p.D == 8 * NC * p.lanes;
    auto mine = [&](int i, float v) { return whole || (i % 8 >= from[i / 8] && i % 8 < to[i / 8]) ? v : 0.0f; };
    constexpr int KEPT = LEAN ? 1 : N;
    float wa[KEPT], wb[KEPT], sa[KEPT], sb[KEPT];
    auto weight = [&](const float* w, int c, int j) { return w && (!TINY || j < to[c]) ? w[at[c] + j] : 0.0f; };
    const float* after = p.after ? p.after + off : nullptr;
    if constexpr (LEAN) {
        for (int i = 0; i < 2 * N; ++i) sums[i * MOST + threadIdx.x] = 0.0f;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            wa[i] = mine(i, weight(after, i / 8, i % 8));
            wb[i] = mine(i, weight(p.before, i / 8, i % 8));
            sa[i] = sb[i] = 0.0f;
        }
    }
    auto wa_of = [&](int i) { if constexpr (LEAN) return mine(i, weight(after, i / 8, i % 8)); else return wa[i]; };
    auto wb_of = [&](int i) { if constexpr (LEAN) return mine(i, weight(p.before, i / 8, i % 8)); else return wb[i]; };
    auto add_a = [&](int i, float v) { if constexpr (LEAN) sums[i * MOST + threadIdx.x] += v; else sa[i] += v; };
    auto add_b = [&](int i, float v) { if constexpr (LEAN) sums[(N + i) * MOST + threadIdx.x] += v; else sb[i] += v; };
    // a lane's places in the row it reads and the row it writes, which go on with the rows
    const int64_t n0 = slot / p.groups, rows_on = p.step / p.groups;
    const T *y_at = (const T*)p.y + n0 * p.ldy + off, *gate_at = (const T*)p.gate + n0 * p.ldg + off, *gh_at = (const T*)p.gh + n0 * p.ldgh + off;
    const S *x_at = (const S*)p.x + n0 * p.ldx + off, *gu_at = (const S*)p.gu + n0 * p.ldgu + off;
    T *h_at = (T*)p.h + n0 * p.ldh + off, *dy_at = (T*)p.dy + n0 * p.lddy + off, *dg_at = (T*)p.dg + n0 * p.lddg + off;
    S *u_at = (S*)p.u + n0 * p.ldu + off, *dx_at = (S*)p.dx + n0 * p.lddx + off;
    auto load_values = [&](NormRow<T, S, NC>& v) {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            load8<TINY>(y_at + at[c], to[c], v.y[c]);
            if (p.gate_kind) load8<TINY>(gate_at + at[c], to[c], v.gate[c]);
            if (p.x) load8<TINY>(x_at + at[c], to[c], v.x[c]);
        }
        y_at += rows_on * p.ldy;
        gate_at += rows_on * p.ldg;
        x_at += rows_on * p.ldx;
    };
    auto load_gradients = [&](NormRow<T, S, NC>& v) {
        if constexpr (GRAD) {
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                if (p.gh) load8<TINY>(gh_at + at[c], to[c], v.gh[c]);
                if (p.gu) load8<TINY>(gu_at + at[c], to[c], v.gu[c]);
            }
            gh_at += rows_on * p.ldgh;
            gu_at += rows_on * p.ldgu;
        }
    };
    NormRow<T, S, NC> now, next;
    if (AHEAD && slot < p.rows) { load_values(next); load_gradients(next); }
    for (int64_t row = slot; row < p.rows; row += p.step) {
        if constexpr (AHEAD) {
            now = next;
            if (row + p.step < p.rows) { load_values(next); load_gradients(next); }
        } else {
            load_values(now);
            if constexpr (!LEAN) load_gradients(now);
        }
        float y[N], u[N], e[N];                               // e: the gate's sigmoid
#pragma unroll
        for (int c = 0; c < NC; ++c) numbers8(now.y[c], y + 8 * c);
#pragma unroll
        for (int i = 0; i < N; ++i) y[i] = mine(i, y[i]);
        float ry = 1.0f;
        if (p.after) ry = normed<N, GROUP>(p, sum, y, mine);
        auto each = [&](auto&& f) {
#pragma unroll
            for (int i = 0; i < N; ++i) f(i);
        };
        each([&](int i) { u[i] = p.after ? y[i] * wa_of(i) : y[i]; });
        float gate[N];
        if (p.gate_kind) {
#pragma unroll
            for (int c = 0; c < NC; ++c) numbers8(now.gate[c], gate + 8 * c);
            if (!whole) each([&](int i) { gate[i] = mine(i, gate[i]); });
            each([&](int i) { e[i] = sigmoid(gate[i]); u[i] *= e[i]; });
            if (p.gate_kind == ACCERL_GATE_SILU) each([&](int i) { u[i] *= gate[i]; });
        }
        each([&](int i) { u[i] *= p.branch; });
        if (p.x)
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                float x[8];
                numbers8(now.x[c], x);
#pragma unroll
                for (int j = 0; j < 8; ++j) u[8 * c + j] += mine(8 * c + j, p.skip * x[j]);
            }
        if constexpr (!GRAD) {
            if (p.u)
#pragma unroll
                for (int c = 0; c < NC; ++c) store8(u_at + at[c], from[c], to[c], u + 8 * c);
            if (p.before) {
                normed<N, GROUP>(p, sum, u, mine);
#pragma unroll
                for (int i = 0; i < N; ++i) u[i] *= wb_of(i);
#pragma unroll
                for (int c = 0; c < NC; ++c) store8(h_at + at[c], from[c], to[c], u + 8 * c);
            }
            u_at += rows_on * p.ldu;
            h_at += rows_on * p.ldh;
        } else {
            float g[N];                                       // the gradient by u
#pragma unroll
            for (int i = 0; i < N; ++i) g[i] = 0.0f;
            if constexpr (LEAN) load_gradients(now);
            if (p.before) {
                const float ru = normed<N, GROUP>(p, sum, u, mine);
                if (p.gh) {
#pragma unroll
                    for (int c = 0; c < NC; ++c) numbers8(now.gh[c], g + 8 * c);
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        g[i] = mine(i, g[i]);
                        add_b(i, g[i] * u[i]);
                        g[i] *= wb_of(i);
                    }
                    through<N, GROUP>(p, sum, g, u, ru);
                }
            }
            if (p.gu)
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    float o[8];
                    numbers8(now.gu[c], o);
#pragma unroll
                    for (int j = 0; j < 8; ++j) g[8 * c + j] += o[j];
                }
            if (p.dx)
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    float o[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) o[j] = p.skip * g[8 * c + j];
                    store8(dx_at + at[c], from[c], to[c], o);
                }
            each([&](int i) { g[i] = mine(i, g[i] * p.branch); });
            if (p.gate_kind) {
                float o[N];
                each([&](int i) { o[i] = g[i] * (p.after ? y[i] * wa_of(i) : y[i]); g[i] *= e[i]; });
                if (p.gate_kind == ACCERL_GATE_SILU) each([&](int i) { o[i] *= e[i] * (1.0f + gate[i] * (1.0f - e[i])); g[i] *= gate[i]; });
                else each([&](int i) { o[i] *= e[i] * (1.0f - e[i]); });
                if (p.dg)
#pragma unroll
                    for (int c = 0; c < NC; ++c) store8(dg_at + at[c], from[c], to[c], o + 8 * c);
            }
            if (p.after) {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    add_a(i, g[i] * y[i]);
                    g[i] *= wa_of(i);
                }
                if (p.dy) through<N, GROUP>(p, sum, g, y, ry);
            }
            if (p.dy)
#pragma unroll
                for (int c = 0; c < NC; ++c) store8(dy_at + at[c], from[c], to[c], g + 8 * c);
            dx_at += rows_on * p.lddx;
            dg_at += rows_on * p.lddg;
            dy_at += rows_on * p.lddy;
        }
    }
    if constexpr (GRAD) {
        // a slot without rows has zeros; slots of a workgroup that have the same weights are added up first
        auto keep = [&](float* out, const float* s, int which) {
            if (!out) return;
            if constexpr (LEAN) {
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    float v[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] = sums[(which * N + 8 * c + j) * MOST + threadIdx.x];
                    store8(out + slot * p.D + at[c], from[c], to[c], v);
                }
            } else if constexpr (GROUP) {
#pragma unroll
                for (int c = 0; c < NC; ++c) store8(out + slot * p.D + at[c], from[c], to[c], s + 8 * c);
            } else {
                const int slots = 256 / p.lanes, nth = threadIdx.x / p.lanes;
                const bool fold = slots % p.groups == 0;
                __syncthreads();
#pragma unroll
                for (int c = 0; c < NC; ++c) store8((fold ? sums + nth * p.D : out + slot * p.D) + at[c], from[c], to[c], s + 8 * c);
                __syncthreads();
                if (fold)
                    for (int i = threadIdx.x; i < p.groups * p.D; i += 256) {
                        float t = 0.0f;
                        for (int k = i / p.D; k < slots; k += p.groups) t += sums[k * p.D + i % p.D];
                        out[(int64_t)blockIdx.x * p.groups * p.D + i] = t;
                    }
            }
        };
        keep(p.da, sa, 0);
        keep(p.db, sb, 1);
    }
}

// The weights' gradients from the workgroups' sums: 64 columns a workgroup, 16 wavefronts take records in turn, joined in 64 bits.
struct NormJoinParams { const float* part[2]; float* out[2]; int64_t records; int D, groups; };
__global__ __launch_bounds__(1024) void block_norm_join_kernel(const NormJoinParams p) {
    __shared__ double red[16][64];
    const int c = blockIdx.x * 64 + (threadIdx.x & 63), w = threadIdx.x >> 6;
    const float* from = p.part[blockIdx.y];
    double s = 0.0;
    if (from && c < p.D * p.groups)
#pragma unroll 4
        for (int64_t k = c / p.D + (int64_t)w * p.groups; k < p.records; k += 16 * p.groups) s += from[k * p.D + c % p.D];
    red[w][threadIdx.x & 63] = s;
    __syncthreads();
    if (from && w == 0 && c < p.D * p.groups) {
        for (int i = 1; i < 16; ++i) s += red[i][threadIdx.x];
        p.out[blockIdx.y][c] = (float)s;
    }
}

int bn_fail(int code, const char* who, const char* what) {
    char msg[160];
    snprintf(msg, sizeof msg, "%s: %s", who, what);
    return set_error(code, msg);
}
int bn_launched(const char* who) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? ACCERL_OK : bn_fail(ACCERL_EHIP, who, hipGetErrorString(e));
}
bool bn_aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

// How rows of d elements (of a group) lie on lanes: nc eights for each of `lanes`; rows a workgroup works on at a time; partial sums of weights it leaves.
struct NormShape { int nc, lanes, threads, at_once; bool group; int64_t blocks, records; };
NormShape bn_shape(int64_t rows, int d, int groups, bool grad) {
    NormShape s{};
    // (forwards, few rows, which are latency alone: one eight a lane, in a workgroup where that takes more than a wavefront.  16 rows of 600, 1024 and 2048, bf16: 4.3, 4.4
    // and 5.5 us, 6.7, 7.6 and 6.0 with two; 1024 rows 6.7, 8.3 and 13.2, and 7.4, 8.4 and 13.8)
    const bool few = !grad && rows <= 1024 && d <= 2048;
    if (d <= (grad || few ? 512 : 1024)) {
        s.nc = d <= 512 ? 1 : 2;
        s.lanes = 1;
        while (s.lanes * 8 * s.nc < d) s.lanes *= 2;
        s.threads = 256;
        s.at_once = 256 / s.lanes;
    } else {
        // (gradients of rows of 600 and 1024 bf16: 470 and 249 us for 2^26 elements with one eight a lane, 496 and 266 with two in a wavefront; of 3000 and 4096:
        // 396 and 250 with two, 656 and 369 with one)
        s.group = true;
        s.nc = few ? 1 : !grad ? 2 : d <= 1024 ? 1 : d <= 8192 ? 2 : 4;
        s.threads = s.lanes = (d + 512 * s.nc - 1) / (512 * s.nc) * 64;
        s.at_once = 1;
    }
    // as many workgroups as are on the chip at once; the slots in all are a multiple of the groups
    const int64_t most = 256 * std::max<int64_t>(1, (grad ? s.nc == 1 ? 768 : 512 : 2048) / s.threads);
    s.blocks = std::max<int64_t>(1, std::min(most, (rows + s.at_once - 1) / s.at_once));
    while (s.blocks * s.at_once % groups) ++s.blocks;
    s.records = s.blocks * (s.at_once % groups == 0 ? groups : s.at_once);
    return s;
}

int bn_sizes(const char* who, int64_t N, int32_t D, int32_t groups) {
    if (N < 0 || D < 1 || groups < 1) return bn_fail(ACCERL_EINVAL, who, "need N >= 0, D >= 1 and groups >= 1");
    if (D % groups) return bn_fail(ACCERL_EINVAL, who, "the channels must be a multiple of the groups");
    if (D > BN_MAX_D || N > ((int64_t)1 << 31)) return bn_fail(ACCERL_EUNSUPPORTED, who, "more than 16384 channels or 2^31 rows");
    return ACCERL_OK;
}

template <typename T, typename S, bool GRAD> void bn_go(const NormParams& p, const NormShape& s, hipStream_t st) {
    const dim3 grid((uint32_t)s.blocks), block(s.threads);
    if (p.D < 8) block_norm_kernel<T, S, 1, 256, false, GRAD, true><<<grid, block, 0, st>>>(p);
    else if (!s.group) {
        if (s.nc == 2) block_norm_kernel<T, S, 2, 256, false, false, false><<<grid, block, 0, st>>>(p);
        else block_norm_kernel<T, S, 1, 256, false, GRAD, false><<<grid, block, 0, st>>>(p);
    } else if (s.nc == 4) {
        block_norm_kernel<T, S, GRAD ? 4 : 2, 512, true, GRAD, false><<<grid, block, 0, st>>>(p);
    } else if (s.nc == 2) {
        if (s.threads <= 256) block_norm_kernel<T, S, 2, 256, true, GRAD, false><<<grid, block, 0, st>>>(p);
        else if (s.threads <= 512) block_norm_kernel<T, S, 2, 512, true, GRAD, false><<<grid, block, 0, st>>>(p);
        else if constexpr (!GRAD) block_norm_kernel<T, S, 2, 1024, true, GRAD, false><<<grid, block, 0, st>>>(p);
    } else {
        block_norm_kernel<T, S, 1, 256, true, GRAD, false><<<grid, block, 0, st>>>(p);
    }
}
template <bool GRAD> int bn_run(const char* who, const accerl_block_norm_args& a, NormParams& p, const NormShape& s, hipStream_t st) {
    const bool wide = a.stream_dtype == ACCERL_DT_F32;
    if (a.dtype == ACCERL_DT_F32) bn_go<float, float, GRAD>(p, s, st);
    else if (a.dtype == ACCERL_DT_BF16) wide ? bn_go<BF16, float, GRAD>(p, s, st) : bn_go<BF16, BF16, GRAD>(p, s, st);
    else wide ? bn_go<F16, float, GRAD>(p, s, st) : bn_go<F16, F16, GRAD>(p, s, st);
    return bn_launched(who);
}

// one table of a call
struct NormTable { const void* p; int64_t ld; bool stream, out; };

// what both calls check, and the parameters they share; `done` is set where nothing is to be done
int bn_check(const char* who, const accerl_block_norm_args* a, const NormTable* tables, int count, bool* done) {
    *done = false;
    if (!a) return bn_fail(ACCERL_EINVAL, who, "NULL argument");
    if (int rc = bn_sizes(who, a->N, a->D, a->groups)) return rc;
    if (!dtype_known(a->dtype) || (a->stream_dtype != a->dtype && a->stream_dtype != ACCERL_DT_F32)) return bn_fail(ACCERL_EINVAL, who, "unknown types, or a residual stream that is neither of the rows' type nor fp32");
    if (a->kind < ACCERL_NORM_RMS || a->kind > ACCERL_NORM_LAYER || a->gate_kind < ACCERL_GATE_NONE || a->gate_kind > ACCERL_GATE_SILU) return bn_fail(ACCERL_EINVAL, who, "unknown kind of norm or gate");
    if (a->groups > 1 && a->before) return bn_fail(ACCERL_EINVAL, who, "groups are for calls without the norm before the next block");
    if (!(a->eps >= FLT_MIN && a->eps < 1e30) || !(a->skip > -1e30 && a->skip < 1e30) || !(a->branch > -1e30 && a->branch < 1e30)) return bn_fail(ACCERL_EINVAL, who, "eps must be positive and normal in fp32, skip and branch finite");
    for (int i = 0; i < count; ++i) if (tables[i].p && tables[i].ld < a->D) return bn_fail(ACCERL_EINVAL, who, "rows overlap (stride < D)");
    if (a->N == 0) { *done = true; return ACCERL_OK; }
    if (!a->y || (a->gate_kind && !a->gate)) return bn_fail(ACCERL_EINVAL, who, "y or the gate is NULL");
    const int e[2] = {dtype_bytes(a->dtype), dtype_bytes(a->stream_dtype)};
    for (int i = 0; i < count; ++i) if (!bn_aligned(tables[i].p, e[tables[i].stream])) return bn_fail(ACCERL_EINVAL, who, "misaligned argument");
    if (!bn_aligned(a->after, 4) || !bn_aligned(a->before, 4)) return bn_fail(ACCERL_EINVAL, who, "misaligned weight");
    for (int i = 0; i < count; ++i)
        for (int j = 0; j < count; ++j) {
            const NormTable &o = tables[i], &t = tables[j];
            if (i == j || !o.out || !o.p || !t.p || (t.out && j < i)) continue;
            const bool over = !t.out && o.p == t.p && (o.ld == t.ld || a->N == 1) && e[o.stream] == e[t.stream];
            if (!over && share(table(o.p, a->N, o.ld, a->D, e[o.stream]), table(t.p, a->N, t.ld, a->D, e[t.stream])))
                return bn_fail(ACCERL_EINVAL, who, "an output overlaps an input (other than lying over it) or another output");
        }
    for (int i = 0; i < count; ++i) {
        const Table o = table(tables[i].p, a->N, tables[i].ld, a->D, e[tables[i].stream]);
        if (tables[i].out && o.at && (share(o, table(a->after, 4 * (int64_t)a->D)) || share(o, table(a->before, 4 * (int64_t)a->D)))) return bn_fail(ACCERL_EINVAL, who, "an output overlaps a weight");
    }
    return ACCERL_OK;
}
// what the weights' gradients and the workspace (of `used` bytes) may lie over: a weight, whole, and nothing
int bn_apart(const char* who, const accerl_block_norm_args& a, const NormTable* tables, int count, int64_t used) {
    const int64_t bytes = 4 * (int64_t)a.D;
    const Table work = table(a.workspace, used), after = table(a.after, bytes), before = table(a.before, bytes), grad_after = table(a.grad_after, bytes), grad_before = table(a.grad_before, bytes);
    for (const Table& g : {grad_after, grad_before}) {
        for (const Table& w : {after, before}) if (g.at != w.at && share(g, w)) return bn_fail(ACCERL_EINVAL, who, "a weight's gradient overlaps a weight (other than lying over it)");
        for (int i = 0; i < count; ++i)
            if (tables[i].p && share(g, table(tables[i].p, a.N, tables[i].ld, a.D, dtype_bytes(tables[i].stream ? a.stream_dtype : a.dtype)))) return bn_fail(ACCERL_EINVAL, who, "a weight's gradient overlaps rows");
    }
    if (share(grad_after, grad_before)) return bn_fail(ACCERL_EINVAL, who, "the weights' gradients overlap");
    bool over = share(work, after) || share(work, before) || share(work, grad_after) || share(work, grad_before);
    for (int i = 0; i < count; ++i) over = over || (tables[i].p && share(work, table(tables[i].p, a.N, tables[i].ld, a.D, dtype_bytes(tables[i].stream ? a.stream_dtype : a.dtype))));
    return over ? bn_fail(ACCERL_EINVAL, who, "the workspace overlaps an input or an output") : ACCERL_OK;
}
NormParams bn_params(const accerl_block_norm_args& a, const NormShape& s) {
    NormParams p{};
    p.y = a.y; p.ldy = a.ld_y;
    p.x = a.x; p.ldx = a.ld_x;
    p.gate = a.gate_kind ? a.gate : nullptr; p.ldg = a.ld_gate;
    p.after = a.after; p.before = a.before;
    p.rows = a.N * a.groups;
    p.step = s.blocks * s.at_once;
    p.D = a.D / a.groups; p.groups = a.groups; p.lanes = s.lanes;
    p.layer = a.kind == ACCERL_NORM_LAYER; p.gate_kind = a.gate_kind;
    p.eps = (float)a.eps; p.skip = (float)a.skip; p.branch = (float)a.branch;
    p.inv_d = (float)(1.0 / p.D);
    return p;
}
int64_t bn_part(const NormShape& s, int d) { return (s.records * d + 3) / 4 * 4; }
}  // namespace
}  // namespace accerl

using namespace accerl;

extern "C" {

int64_t accerl_block_norm_workspace(int64_t N, int32_t D, int32_t groups) {
    if (int rc = bn_sizes("block_norm_workspace", N, D, groups)) return rc;
    return 2 * 4 * bn_part(bn_shape(N * groups, D / groups, groups, true), D / groups);
}

int accerl_block_norm(const accerl_block_norm_args* a, void* stream) {
    const char* who = "block_norm";
    bool done;
    NormTable t[5] = {};
    if (a) {
        const NormTable all[5] = {{a->y, a->ld_y, false, false}, {a->x, a->ld_x, true, false}, {a->gate_kind ? a->gate : nullptr, a->ld_gate, false, false},
                                  {a->out_u, a->ld_u, true, true}, {a->before ? a->out_h : nullptr, a->ld_h, false, true}};
        std::copy(all, all + 5, t);
    }
    if (int rc = bn_check(who, a, t, 5, &done)) return rc;
    if (done) return ACCERL_OK;
    if (a->before ? !a->out_h : !a->out_u) return bn_fail(ACCERL_EINVAL, who, "NULL output");
    const NormShape s = bn_shape(a->N * a->groups, a->D / a->groups, a->groups, false);
    NormParams p = bn_params(*a, s);
    p.u = a->out_u; p.ldu = a->ld_u;
    p.h = a->out_h; p.ldh = a->ld_h;
    return bn_run<false>(who, *a, p, s, (hipStream_t)stream);
}

int accerl_block_norm_grad(const accerl_block_norm_args* a, void* stream) {
    const char* who = "block_norm_grad";
    bool done;
    NormTable t[8] = {};
    if (a) {
        const NormTable all[8] = {{a->y, a->ld_y, false, false}, {a->x, a->ld_x, true, false}, {a->gate_kind ? a->gate : nullptr, a->ld_gate, false, false},
                                  {a->grad_u, a->ld_grad_u, true, false}, {a->before ? a->grad_h : nullptr, a->ld_grad_h, false, false},
                                  {a->grad_y, a->ld_grad_y, false, true}, {a->grad_x, a->ld_grad_x, true, true}, {a->grad_gate, a->ld_grad_gate, false, true}};
        std::copy(all, all + 8, t);
    }
    if (int rc = bn_check(who, a, t, 8, &done)) return rc;
    if ((a->grad_after && !a->after) || (a->grad_before && !a->before) || (a->grad_x && !a->x && a->N) || (a->grad_gate && !a->gate_kind))
        return bn_fail(ACCERL_EINVAL, who, "a gradient by what the call does not have");
    if (!bn_aligned(a->grad_after, 4) || !bn_aligned(a->grad_before, 4)) return bn_fail(ACCERL_EINVAL, who, "misaligned argument");
    const bool sums = a->grad_after || a->grad_before;
    const NormShape s = bn_shape(a->N * a->groups, a->D / a->groups, a->groups, true);
    const int64_t part = bn_part(s, a->D / a->groups);
    float* ws = (float*)a->workspace;
    if (sums) {
        if (!ws || !bn_aligned(ws, 16)) return bn_fail(ACCERL_EINVAL, who, "workspace is NULL or misaligned");
        if (a->workspace_bytes < 8 * part) return bn_fail(ACCERL_EINVAL, who, "workspace smaller than accerl_block_norm_workspace says");
        if (int rc = bn_apart(who, *a, t, 8, 8 * part)) return rc;
    }
    if (done && !sums) return ACCERL_OK;
    NormParams p = bn_params(*a, s);
    p.gu = a->grad_u; p.ldgu = a->ld_grad_u;
    p.gh = a->before ? a->grad_h : nullptr; p.ldgh = a->ld_grad_h;
    p.dy = a->grad_y; p.lddy = a->ld_grad_y;
    p.dx = a->grad_x; p.lddx = a->ld_grad_x;
    p.dg = a->grad_gate; p.lddg = a->ld_grad_gate;
    p.da = a->grad_after ? ws : nullptr;
    p.db = a->grad_before ? ws + part : nullptr;
    if (int rc = bn_run<true>(who, *a, p, s, (hipStream_t)stream)) return rc;        // (no rows: the sums become zeros)
    if (!sums) return ACCERL_OK;
    NormJoinParams j{};
    j.part[0] = p.da; j.out[0] = a->grad_after;
    j.part[1] = p.db; j.out[1] = a->grad_before;
    j.records = s.records; j.D = p.D; j.groups = a->groups;
    block_norm_join_kernel<<<dim3((a->D + 63) / 64, 2), dim3(1024), 0, (hipStream_t)stream>>>(j);
    return bn_launched(who);
}

}  // extern "C"
