// The norms around a block with its gate and its residual, and their gradients.
//
// A row is read once and stays in the registers of its lanes, eight neighbouring elements at a time: all statistics are taken from there, the mean
// first and then the squares around it.  Bound by memory: the gradients' six sums over a row lie between one row's loads and its stores, so that several
// rows have to be under way on a compute unit.  Rows of up to 1024 elements belong to a part of a wavefront or to a whole one, longer rows to a workgroup.
#include <algorithm>
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
    float *da, *db;                       // partial sums of the weights' gradients, [slot][D of a group]
    int64_t rows;                         // rows x groups
    int64_t step;                         // from a slot's row to its next: a multiple of the groups, so that a slot keeps its weights
    int D, groups, lanes;                 // of a group's row; lanes a row has
    int layer, gate_kind;
    float eps, skip, branch, inv_d;
};

// eight elements of a row, of which `left` are inside (the others 0)
template <typename T> __device__ __forceinline__ void load8(const T* p, int left, float* o) {
    if (left >= 8) {
        if constexpr (sizeof(T) == 4) {
            const v4f a = __builtin_bit_cast(v4f, *(const u32x4_at4*)p), b = __builtin_bit_cast(v4f, *(const u32x4_at4*)(p + 4));
#pragma unroll
            for (int j = 0; j < 4; ++j) { o[j] = a[j]; o[4 + j] = b[j]; }
        } else {
            const u32x4 w = *(const u32x4_at2*)p;
#pragma unroll
            for (int j = 0; j < 4; ++j) el_pair<T>(w[j], o[2 * j], o[2 * j + 1]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = j < left ? el_f32(p[j]) : 0.0f;
    }
}
template <typename T> __device__ __forceinline__ void store8(T* p, int left, const float* v) {
    if (left >= 8) {
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
        for (int j = 0; j < 8; ++j) if (j < left) p[j] = f32_el<T>(v[j]);
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

__device__ __forceinline__ float sigmoid(float x) { return 1.0f / (1.0f + __expf(-x)); }

// z -> (z - mean) and the reciprocal root; elements behind the row's end stay 0
template <int N, bool GROUP> __device__ __forceinline__ float normed(const NormParams& p, RowSum<GROUP>& sum, float* z, const int* left) {
    if (p.layer) {
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) s += z[i];
        const float mean = sum(s) * p.inv_d;
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = i % 8 < left[i / 8] ? z[i] - mean : 0.0f;
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

template <typename T, typename S, int NC, bool GROUP, bool GRAD>
__global__ __launch_bounds__(GROUP ? 1024 : 256) void block_norm_kernel(const NormParams p) {
    constexpr int N = 8 * NC;
    __shared__ float red[2][16][2];
    RowSum<GROUP> sum{red, p.lanes};
    const int lane = GROUP ? threadIdx.x : threadIdx.x & (p.lanes - 1);
    const int64_t slot = GROUP ? blockIdx.x : (int64_t)blockIdx.x * (256 / p.lanes) + threadIdx.x / p.lanes;
    const int part = (int)(slot % p.groups);
    int at[NC], left[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        at[c] = (c * p.lanes + lane) * 8;
        left[c] = min(max(p.D - at[c], 0), 8);
        if (!left[c]) at[c] = 0;
    }
    float wa[N], wb[N], sa[N], sb[N];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            wa[8 * c + j] = p.after && j < left[c] ? p.after[part * p.D + at[c] + j] : 0.0f;
            wb[8 * c + j] = p.before && j < left[c] ? p.before[at[c] + j] : 0.0f;
            sa[8 * c + j] = sb[8 * c + j] = 0.0f;
        }
    }
    for (int64_t row = slot; row < p.rows; row += p.step) {
        const int64_t n = p.groups == 1 ? row : row / p.groups;
        const int off = part * p.D;
        float y[N], gt[N], u[N];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            load8((const T*)p.y + n * p.ldy + off + at[c], left[c], y + 8 * c);
            if (p.gate_kind) load8((const T*)p.gate + n * p.ldg + off + at[c], left[c], gt + 8 * c);
            if (p.x) load8((const S*)p.x + n * p.ldx + off + at[c], left[c], u + 8 * c);
        }
        float gu[N], gh[N];
        if constexpr (GRAD) {
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                if (p.gu) load8((const S*)p.gu + n * p.ldgu + off + at[c], left[c], gu + 8 * c);
                if (p.gh) load8((const T*)p.gh + n * p.ldgh + off + at[c], left[c], gh + 8 * c);
            }
#pragma unroll
            for (int i = 0; i < N; ++i) { if (!p.gu) gu[i] = 0.0f; if (!p.gh) gh[i] = 0.0f; }
        }
        float ry = 1.0f;
        if (p.after) ry = normed<N, GROUP>(p, sum, y, left);
        // u, and with gradients the gate's value (in gt) and its slope
        float slope[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float m = p.after ? y[i] * wa[i] : y[i];
            float s = 1.0f;
            slope[i] = 0.0f;
            if (p.gate_kind) {
                const float e = sigmoid(gt[i]);
                s = p.gate_kind == ACCERL_GATE_SIGMOID ? e : gt[i] * e;
                slope[i] = p.gate_kind == ACCERL_GATE_SIGMOID ? e * (1.0f - e) : e * (1.0f + gt[i] * (1.0f - e));
            }
            gt[i] = s;
            u[i] = p.branch * s * m + (p.x ? p.skip * u[i] : 0.0f);
            if (i % 8 >= left[i / 8]) u[i] = 0.0f;
        }
        if constexpr (!GRAD) {
            if (p.u)
#pragma unroll
                for (int c = 0; c < NC; ++c) store8((S*)p.u + n * p.ldu + off + at[c], left[c], u + 8 * c);
            if (p.before) {
                normed<N, GROUP>(p, sum, u, left);
#pragma unroll
                for (int i = 0; i < N; ++i) u[i] *= wb[i];
#pragma unroll
                for (int c = 0; c < NC; ++c) store8((T*)p.h + n * p.ldh + off + at[c], left[c], u + 8 * c);
            }
        } else {
            if (p.before) {
                const float ru = normed<N, GROUP>(p, sum, u, left);
                float t[N];
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    sb[i] += gh[i] * u[i];
                    t[i] = gh[i] * wb[i];
                }
                through<N, GROUP>(p, sum, t, u, ru);
#pragma unroll
                for (int i = 0; i < N; ++i) gu[i] += t[i];
            }
            float o[N];
            if (p.dx) {
#pragma unroll
                for (int i = 0; i < N; ++i) o[i] = p.skip * gu[i];
#pragma unroll
                for (int c = 0; c < NC; ++c) store8((S*)p.dx + n * p.lddx + off + at[c], left[c], o + 8 * c);
            }
#pragma unroll
            for (int i = 0; i < N; ++i) gu[i] *= p.branch;
            if (p.dg) {
#pragma unroll
                for (int i = 0; i < N; ++i) o[i] = gu[i] * (p.after ? y[i] * wa[i] : y[i]) * slope[i];
#pragma unroll
                for (int c = 0; c < NC; ++c) store8((T*)p.dg + n * p.lddg + off + at[c], left[c], o + 8 * c);
            }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                gu[i] *= gt[i];
                if (i % 8 >= left[i / 8]) gu[i] = 0.0f;
            }
            if (p.after) {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    sa[i] += gu[i] * y[i];
                    gu[i] *= wa[i];
                }
                if (p.dy) through<N, GROUP>(p, sum, gu, y, ry);
            }
            if (p.dy)
#pragma unroll
                for (int c = 0; c < NC; ++c) store8((T*)p.dy + n * p.lddy + off + at[c], left[c], gu + 8 * c);
        }
    }
    if constexpr (GRAD) {
        // a slot without rows has zeros
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            if (p.da) store8(p.da + slot * p.D + at[c], left[c], sa + 8 * c);
            if (p.db) store8(p.db + slot * p.D + at[c], left[c], sb + 8 * c);
        }
    }
}

// The weights' gradients from the slots' sums: 64 columns a workgroup, 16 wavefronts take slots in turn, joined in 64 bits.
struct NormJoinParams { const float* part[2]; float* out[2]; int64_t slots; int D, groups; };
__global__ __launch_bounds__(1024) void block_norm_join_kernel(const NormJoinParams p) {
    __shared__ double red[16][64];
    const int c = blockIdx.x * 64 + (threadIdx.x & 63), w = threadIdx.x >> 6;
    const float* from = p.part[blockIdx.y];
    double s = 0.0;
    if (from && c < p.D * p.groups)
        for (int64_t k = c / p.D + (int64_t)w * p.groups; k < p.slots; k += 16 * p.groups) s += from[k * p.D + c % p.D];
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

// How rows of d elements (of a group) lie on lanes: nc eights for each of `lanes`; rows a workgroup works on at a time.
struct NormShape { int nc, lanes, threads, at_once; bool group; int64_t blocks; };
NormShape bn_shape(int64_t rows, int d, int groups) {
    NormShape s{};
    if (d <= 1024) {
        s.nc = d <= 512 ? 1 : 2;
        s.lanes = 1;
        while (s.lanes * 8 * s.nc < d) s.lanes *= 2;
        s.threads = 256;
        s.at_once = 256 / s.lanes;
    } else {
        s.group = true;
        s.nc = 2;
        s.threads = s.lanes = (d + 1023) / 1024 * 64;
        s.at_once = 1;
    }
    // two workgroups of 1024 lanes a compute unit; the slots in all are a multiple of the groups
    int64_t most = 256 * 2048 / s.threads;
    s.blocks = std::max<int64_t>(1, std::min(most, (rows + s.at_once - 1) / s.at_once));
    while (s.blocks * s.at_once % groups) ++s.blocks;
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
    if (s.group) block_norm_kernel<T, S, 2, true, GRAD><<<grid, block, 0, st>>>(p);
    else if (s.nc == 2) block_norm_kernel<T, S, 2, false, GRAD><<<grid, block, 0, st>>>(p);
    else block_norm_kernel<T, S, 1, false, GRAD><<<grid, block, 0, st>>>(p);
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
    if (!(a->eps > 0.0 && a->eps < 1e30) || !(a->skip > -1e30 && a->skip < 1e30) || !(a->branch > -1e30 && a->branch < 1e30)) return bn_fail(ACCERL_EINVAL, who, "eps must be positive, skip and branch finite");
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
    return ACCERL_OK;
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
int64_t bn_part(const NormShape& s, int d) { return (s.blocks * s.at_once * d + 3) / 4 * 4; }
}  // namespace
}  // namespace accerl

using namespace accerl;

extern "C" {

int64_t accerl_block_norm_workspace(int64_t N, int32_t D, int32_t groups) {
    if (int rc = bn_sizes("block_norm_workspace", N, D, groups)) return rc;
    return 2 * 4 * bn_part(bn_shape(N * groups, D / groups, groups), D / groups);
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
    const NormShape s = bn_shape(a->N * a->groups, a->D / a->groups, a->groups);
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
    const NormShape s = bn_shape(a->N * a->groups, a->D / a->groups, a->groups);
    const int64_t part = bn_part(s, a->D / a->groups);
    float* ws = (float*)a->workspace;
    if (sums) {
        if (!ws || !bn_aligned(ws, 16)) return bn_fail(ACCERL_EINVAL, who, "workspace is NULL or misaligned");
        if (a->workspace_bytes < 8 * part) return bn_fail(ACCERL_EINVAL, who, "workspace smaller than accerl_block_norm_workspace says");
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
    j.slots = s.blocks * s.at_once; j.D = p.D; j.groups = a->groups;
    block_norm_join_kernel<<<dim3((a->D + 63) / 64, 2), dim3(1024), 0, (hipStream_t)stream>>>(j);
    return bn_launched(who);
}

}  // extern "C"
