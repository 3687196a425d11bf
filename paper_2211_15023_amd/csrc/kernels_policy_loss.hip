// Clipped policy loss with a KL term and an entropy term over wide action sets, its gradient, and the log-probabilities of actions.
// With z the logits of a row, z' the reference policy's, p = softmax(z), l = logsumexp(z), a the action:
//   lp = z_a - l,  r = exp(lp - old),  L = -min(r A, clip(r, 1 - lo, 1 + hi) A) + ck KL - ch H,  H = -sum p log p,
//   KL = sum p' log(p' / p) | sum p log(p / p') | exp(lr - lp) - (lr - lp) - 1.
// The gradient has one form for all of them, with coefficients that are the row's:
//   dL/dz_j = p_j (c0 + c1 (z_j - m) + c2 (z_j - z'_j)) - c3 p'_j + ca [j = a].
// One pass over a row gives the maxima m, m' and sums under them (of exp(z - m), exp(z - m) (z - m), exp(z' - m') and
// exp(z' - m') (z' - z) or exp(z - m) (z - z')), corrected where a maximum grows; a second pass writes the gradient.
#include <float.h>
#include <stdio.h>

#include <type_traits>

#include "wide_ops.h"

namespace accerl {
namespace {

constexpr int64_t PL_MAX_A = 1 << 20;
constexpr int PL_RECORDS = 2048;          // workgroups of a row pass, each leaves one record of sums
constexpr int PL_PARTS = 2048;            // pieces of rows, where a row is split
constexpr float PL_LOG2E = 1.44269504088896340736f;

struct RowSum { float m, s, u, mr, sr, t; };
struct Part { RowSum r; float za, pad; };      // za: the action's logit, in the piece that holds it
struct Record { double loss, kl, ent, clipped; };

struct LossParams {
    const void* z; const void* zr; void* g;
    const uint8_t* mask;
    const int32_t* act;
    const float *old, *adv, *w, *ref_lp;
    float *loss, *lp, *kl, *ent;
    Record* rec;
    Part* part;
    int64_t B, ldz, ldr, ldg, ldm;
    int A, kind;             // accerl_kl_kind
    int only_lp;             // log-probabilities and entropies only
    int splits, chunk;       // pieces of a row, elements of a piece
    double lo, hi;           // the clipping borders themselves
    float ck, ch, scale;
};

// what a row's gradient and outputs need
struct Coef { float m, inv_s, mr, inv_sr, c0, c1, c2, c3, ca; int zero; };

__device__ __forceinline__ float pl_exp(float d) { return __builtin_amdgcn_exp2f(d * PL_LOG2E); }   // d <= 0: results below 2^-126 may be 0
__device__ __forceinline__ RowSum row_empty() { return {-FLT_MAX, 0.0f, 0.0f, -FLT_MAX, 0.0f, 0.0f}; }

// Sums under a larger maximum.  The difference of maxima is kept finite so that an empty side's zeros stay zeros.
template <int KL>
__device__ __forceinline__ void row_raise(RowSum& a, float m, float mr) {
    const float d = fmaxf(a.m - m, -FLT_MAX), f = pl_exp(d);
    a.u = f * (a.u + a.s * d);
    a.s *= f;
    if constexpr (KL == 2) a.t *= f;
    a.m = m;
    if constexpr (KL != 0) {
        const float fr = pl_exp(fmaxf(a.mr - mr, -FLT_MAX));
        a.sr *= fr;
        if constexpr (KL == 1) a.t *= fr;
        a.mr = mr;
    }
}
template <int KL>
__device__ __forceinline__ RowSum row_join(RowSum a, RowSum b) {
    const float m = fmaxf(a.m, b.m), mr = fmaxf(a.mr, b.mr);
    row_raise<KL>(a, m, mr);
    row_raise<KL>(b, m, mr);
    a.s += b.s; a.u += b.u; a.sr += b.sr; a.t += b.t;
    return a;
}
// The sums take one element.  Its probability decides whether its logit counts: masked places are -inf, and 0 * inf is no part of a sum.
template <int KL>
__device__ __forceinline__ void row_add(RowSum& a, float z, float zr) {
    const float d = z - a.m, e = pl_exp(d);
    a.s += e;
    a.u = fmaf(e, fmaxf(d, -1000.0f), a.u);
    if constexpr (KL != 0) {
        const float er = pl_exp(zr - a.mr);
        a.sr += er;
        if constexpr (KL == 1) a.t = fmaf(er, er > 0.0f ? zr - z : 0.0f, a.t);
        else a.t = fmaf(e, e > 0.0f ? z - zr : 0.0f, a.t);
    }
}
template <int KL>
__device__ __forceinline__ RowSum row_shuffle(RowSum a, int lanes) {
    for (int o = lanes >> 1; o > 0; o >>= 1) {
        RowSum b;
        b.m = __shfl_xor(a.m, o); b.s = __shfl_xor(a.s, o); b.u = __shfl_xor(a.u, o);
        b.mr = b.sr = b.t = 0.0f;
        if constexpr (KL != 0) { b.mr = __shfl_xor(a.mr, o); b.sr = __shfl_xor(a.sr, o); b.t = __shfl_xor(a.t, o); }
        a = row_join<KL>(a, b);
    }
    return a;
}

// the gradient at one element
template <int KL>
__device__ __forceinline__ float grad_at(const Coef& c, float z, float zr) {
    const float d = z - c.m, p = pl_exp(d) * c.inv_s;
    float t = fmaf(c.c1, fmaxf(d, -1000.0f), c.c0);
    if constexpr (KL == 2) t = fmaf(c.c2, p == 0.0f ? 0.0f : fminf(z - zr, FLT_MAX), t);
    t *= p;
    if constexpr (KL == 1) t = fmaf(-c.c3, pl_exp(zr - c.mr) * c.inv_sr, t);
    return t;
}

struct RowOut { float loss, lp, kl, ent, clipped; };

__device__ __forceinline__ float pl_log(float x) { return logf(x); }
__device__ __forceinline__ double pl_log(double x) { return log(x); }
__device__ __forceinline__ float pl_log_ratio(float a, float b) {        // log(a / b), exact to its own size where a is close to b
    const float q = a / b;
    return q > 0.5f && q < 2.0f ? log1pf((a - b) / b) : logf(q);
}
__device__ __forceinline__ double pl_log_ratio(double a, double b) { return log(a / b); }
__device__ __forceinline__ float pl_exp_full(float x) { return expf(x); }
__device__ __forceinline__ double pl_exp_full(double x) { return exp(x); }

// Scalars of a row from its sums.  R: float where a wavefront holds many rows, double where the row is long and a wavefront does it once.
// The ratio may be replaced (`ratio`, a double) by one that was worked out more exactly.
template <int KL, typename R>
__device__ __forceinline__ void row_finish(const LossParams& p, const RowSum& q, int64_t row, float za, const double* ratio, Coef& c, RowOut& o) {
    const bool empty = q.s == 0.0f;
    const R ls = pl_log((R)q.s), lp = ((R)za - (R)q.m) - ls, ent = ls - (R)q.u / (R)q.s;
    c.m = q.m; c.mr = q.mr; c.inv_s = (float)((R)1 / (R)q.s); c.inv_sr = q.sr == 0.0f ? 0.0f : (float)((R)1 / (R)q.sr);
    c.zero = empty;
    o.lp = empty ? -INFINITY : (float)lp;
    o.ent = empty ? 0.0f : (float)ent;
    o.loss = o.kl = o.clipped = 0.0f;
    if (p.only_lp) return;
    const float w = p.w ? p.w[row] : 1.0f, adv = p.adv[row];
    const R r = ratio ? (R)*ratio : lp == (R)-INFINITY ? (R)0 : pl_exp_full(lp - (R)p.old[row]);
    const bool above = ratio ? *ratio > p.hi : r > (R)p.hi, below = ratio ? *ratio < p.lo : r < (R)p.lo;
    const bool cut = adv >= 0.0f ? above : below;
    const R pg = cut ? -(adv >= 0.0f ? (R)p.hi : (R)p.lo) * (R)adv : -r * (R)adv;
    R at = cut ? (R)0 : -r * (R)adv, kl = 0, c0 = 0, c2 = 0, c3 = 0;
    const R ck = p.ck, ch = p.ch;
    if constexpr (KL == 0) {
        if (p.kind == ACCERL_KL_SAMPLED) {
            const R d = (R)p.ref_lp[row] - lp, e = pl_exp_full(d);
            kl = d == (R)INFINITY ? d : e - d - (R)1;
            if (ck != (R)0) at += ck * ((R)1 - e);
        }
    } else {
        const R dl = ((R)q.m - (R)q.mr) + pl_log_ratio((R)q.s, (R)q.sr);       // l - l'
        if constexpr (KL == 1) {
            if (q.sr != 0.0f) { kl = (R)q.t / (R)q.sr + dl; c0 = ck; c3 = ck; }
        } else {
            kl = q.sr == 0.0f ? (R)INFINITY : (R)q.t / (R)q.s - dl;
            if (ck != (R)0) c0 = -ck * (dl + kl);
            c2 = ck;
        }
    }
    const R by = (R)w * (R)p.scale;
    c.c0 = (float)(by * (c0 - at + ch * (ent - ls)));
    c.c1 = (float)(by * ch);
    c.c2 = (float)(by * c2);
    c.c3 = (float)(by * c3);
    c.ca = (float)(by * at);
    if (empty) { o.ent = 0.0f; return; }
    o.kl = (float)kl;
    o.loss = (float)(pg + (ck == (R)0 ? (R)0 : ck * kl) - ch * ent);
    o.clipped = above || below ? 1.0f : 0.0f;
}

__device__ __forceinline__ bool row_dead(const LossParams& p, int64_t row) {
    const int a = p.act[row];
    return a < 0 || a >= p.A || (!p.only_lp && p.w && p.w[row] == 0.0f);
}
__device__ __forceinline__ void row_store(const LossParams& p, int64_t row, const RowOut& o) {
    if (p.loss) p.loss[row] = o.loss;
    if (p.lp) p.lp[row] = o.lp;
    if (p.kl) p.kl[row] = o.kl;
    if (p.ent) p.ent[row] = o.ent;
}
__device__ __forceinline__ void rec_add(const LossParams& p, Record& r, int64_t row, const RowOut& o) {
    const double w = p.w ? p.w[row] : 1.0;
    r.loss += w * o.loss; r.kl += w * o.kl; r.ent += w * o.ent; r.clipped += w * o.clipped;
}

// ---------------------------------------------------------------- narrow rows: several lanes of a wavefront hold one
// G lanes hold a row, lane j its elements j, j + G, ..  (E of them at most).  A wavefront does 64 / G rows at a time.
constexpr int NR_THREADS = 256;
template <typename T, int KL, int E>
__global__ __launch_bounds__(NR_THREADS) void loss_narrow_kernel(const LossParams p, int G) {
    __shared__ Record s_rec[NR_THREADS / 64];
    const int tid = threadIdx.x, j = tid & (G - 1);
    const int rows = NR_THREADS / G;
    Record rec = {0, 0, 0, 0};
    for (int64_t row = (int64_t)blockIdx.x * rows + tid / G; row < p.B; row += (int64_t)gridDim.x * rows) {
        RowOut o = {0, 0, 0, 0, 0};
        T* g = p.g ? (T*)p.g + row * p.ldg : nullptr;
        if (row_dead(p, row)) {
            if (g)
                for (int i = j; i < p.A; i += G) g[i] = f32_el<T>(0.0f);
            if (j == 0) row_store(p, row, o);
            continue;
        }
        const T* z = (const T*)p.z + row * p.ldz;
        const T* zr = KL ? (const T*)p.zr + row * p.ldr : nullptr;
        const uint8_t* mask = p.mask ? p.mask + row * p.ldm : nullptr;
        float a[E], b[E];
        RowSum q = row_empty();
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const int at = j + i * G;
            const bool in = at < p.A && (!mask || mask[at]);
            a[i] = in ? el_f32(z[at]) : -INFINITY;
            b[i] = KL && in ? el_f32(zr[at]) : -INFINITY;
            q.m = fmaxf(q.m, a[i]);
            q.mr = fmaxf(q.mr, b[i]);
        }
        for (int k = G >> 1; k > 0; k >>= 1) {
            q.m = fmaxf(q.m, __shfl_xor(q.m, k));
            if constexpr (KL != 0) q.mr = fmaxf(q.mr, __shfl_xor(q.mr, k));
        }
#pragma unroll
        for (int i = 0; i < E; ++i) row_add<KL>(q, a[i], b[i]);
        for (int k = G >> 1; k > 0; k >>= 1) {
            q.s += __shfl_xor(q.s, k);
            q.u += __shfl_xor(q.u, k);
            if constexpr (KL != 0) { q.sr += __shfl_xor(q.sr, k); q.t += __shfl_xor(q.t, k); }
        }
        const int act = p.act[row];
        const float za = mask && !mask[act] ? -INFINITY : el_f32(z[act]);
        Coef c;
        double ratio;
        const double* better = nullptr;
        if (!p.only_lp && q.s > 0.0f) {
            // Next to a clipping border the side decides over the whole gradient: there the sum is taken again in 64 bits.  (All lanes of
            // a row branch alike; the 32-bit ratio is off by a few parts in 2^24.)
            const float r = expf(za - q.m - logf(q.s) - p.old[row]);
            if (fabsf(r - (float)p.hi) < 4e-6f * r || fabsf(r - (float)p.lo) < 4e-6f * r) {
                double s = 0.0;
#pragma unroll
                for (int i = 0; i < E; ++i) s += exp((double)a[i] - (double)q.m);
                for (int k = G >> 1; k > 0; k >>= 1) s += __shfl_xor(s, k);
                ratio = exp((double)za - (double)q.m - log(s) - (double)p.old[row]);
                better = &ratio;
            }
        }
        row_finish<KL, float>(p, q, row, za, better, c, o);
        if (g) {
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const int at = j + i * G;
                if (at >= p.A) break;
                float v = grad_at<KL>(c, a[i], b[i]);
                if (at == act) v += c.ca;
                g[at] = f32_el<T>(c.zero ? 0.0f : v);
            }
        }
        if (j == 0) {
            row_store(p, row, o);
            if (p.rec) rec_add(p, rec, row, o);
        }
    }
    if (!p.rec) return;
    for (int k = 32; k > 0; k >>= 1) {
        rec.loss += __shfl_xor(rec.loss, k); rec.kl += __shfl_xor(rec.kl, k);
        rec.ent += __shfl_xor(rec.ent, k); rec.clipped += __shfl_xor(rec.clipped, k);
    }
    if ((tid & 63) == 0) s_rec[tid >> 6] = rec;
    __syncthreads();
    if (tid == 0) {
        for (int k = 1; k < NR_THREADS / 64; ++k) {
            rec.loss += s_rec[k].loss; rec.kl += s_rec[k].kl; rec.ent += s_rec[k].ent; rec.clipped += s_rec[k].clipped;
        }
        p.rec[blockIdx.x] = rec;
    }
}

// ---------------------------------------------------------------- wide rows: a workgroup holds one, or a piece of one
constexpr int WR_THREADS = 512;
constexpr int WR_WAVES = WR_THREADS / 64;

// A vector of 16 bytes of a row from element i on as floats; past the end, and where the mask has a zero, -inf.
template <typename T, int VEC>
__device__ __forceinline__ void load_vec(const T* row, const uint8_t* mask, int i, int end, float (&v)[VEC]) {
    if (i + VEC <= end) {
        if constexpr (VEC == 4) {
            const u32x4 w = *(const u32x4_at4*)(row + i);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = __uint_as_float(w[e]);
        } else {
            const u32x4 w = *(const u32x4_at2*)(row + i);
#pragma unroll
            for (int e = 0; e < 4; ++e) el_pair<T>(w[e], v[2 * e], v[2 * e + 1]);
        }
        if (mask) {
#pragma unroll
            for (int k = 0; k < VEC / 4; ++k) {
                typedef uint32_t u32_at1 __attribute__((aligned(1)));
                const uint32_t w = *(const u32_at1*)(mask + i + 4 * k);
#pragma unroll
                for (int e = 0; e < 4; ++e) if (!((w >> (8 * e)) & 0xffu)) v[4 * k + e] = -INFINITY;
            }
        }
    } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[e] = i + e < end && (!mask || mask[i + e]) ? el_f32(row[i + e]) : -INFINITY;
    }
}
template <typename T, int VEC>
__device__ __forceinline__ void store_vec(T* row, int i, int end, const float (&v)[VEC]) {
    if (i + VEC <= end) {
        if constexpr (VEC == 4) {
            typedef v4f v4f_at4 __attribute__((aligned(4)));
            *(v4f_at4*)(row + i) = (v4f){v[0], v[1], v[2], v[3]};
        } else {
            u32x4 w;
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = f32_pair<T>(v[2 * e], v[2 * e + 1]);
            *(u32x4_at2*)(row + i) = w;
        }
    } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) if (i + e < end) row[i + e] = f32_el<T>(v[e]);
    }
}

template <typename T, int KL>
__device__ __forceinline__ RowSum wide_sum(const T* z, const T* zr, const uint8_t* mask, int first, int end) {
    constexpr int VEC = 16 / sizeof(T);
    RowSum q = row_empty();
    for (int i = first + (int)threadIdx.x * VEC; i < end; i += WR_THREADS * VEC) {
        float a[VEC], b[VEC];
        load_vec<T, VEC>(z, mask, i, end, a);
        if constexpr (KL != 0) load_vec<T, VEC>(zr, mask, i, end, b);
        float m = q.m, mr = q.mr;
#pragma unroll
        for (int e = 0; e < VEC; ++e) { m = fmaxf(m, a[e]); if constexpr (KL != 0) mr = fmaxf(mr, b[e]); }
        row_raise<KL>(q, m, mr);
#pragma unroll
        for (int e = 0; e < VEC; ++e) row_add<KL>(q, a[e], KL ? b[e] : 0.0f);
    }
    return row_shuffle<KL>(q, 64);
}
// the sums of the workgroup's wavefronts, in wavefront 0 (all of its lanes)
template <int KL>
__device__ __forceinline__ RowSum wide_join(RowSum q, RowSum (&s)[WR_WAVES]) {
    const int lane = threadIdx.x & 63;
    if (lane == 0) s[threadIdx.x >> 6] = q;
    __syncthreads();
    return row_shuffle<KL>(s[lane & (WR_WAVES - 1)], WR_WAVES);
}
template <typename T>
__device__ __forceinline__ void wide_zero(T* g, int first, int end) {
    constexpr int VEC = 16 / sizeof(T);
    float v[VEC] = {};
    for (int i = first + (int)threadIdx.x * VEC; i < end; i += WR_THREADS * VEC) store_vec<T, VEC>(g, i, end, v);
}
template <typename T, int KL>
__device__ __forceinline__ void wide_grad(const LossParams& p, const Coef& c, int act, const T* z, const T* zr, const uint8_t* mask, T* g, int first, int end) {
    constexpr int VEC = 16 / sizeof(T);
    for (int i = first + (int)threadIdx.x * VEC; i < end; i += WR_THREADS * VEC) {
        float a[VEC], b[VEC];
        load_vec<T, VEC>(z, mask, i, end, a);
        if constexpr (KL != 0) load_vec<T, VEC>(zr, mask, i, end, b);
#pragma unroll
        for (int e = 0; e < VEC; ++e) a[e] = grad_at<KL>(c, a[e], KL ? b[e] : 0.0f);
        if ((unsigned)(act - i) < (unsigned)VEC) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) a[e] += act - i == e ? c.ca : 0.0f;
        }
        store_vec<T, VEC>(g, i, end, a);
    }
}

// Rows one after the other, each by the whole workgroup.
template <typename T, int KL>
__global__ __launch_bounds__(WR_THREADS) void loss_wide_kernel(const LossParams p) {
    __shared__ RowSum s_sum[WR_WAVES];
    __shared__ Coef s_coef;
    Record rec = {0, 0, 0, 0};
    for (int64_t row = blockIdx.x; row < p.B; row += gridDim.x) {
        RowOut o = {0, 0, 0, 0, 0};
        T* g = p.g ? (T*)p.g + row * p.ldg : nullptr;
        if (row_dead(p, row)) {
            if (g) wide_zero<T>(g, 0, p.A);
            if (threadIdx.x == 0) row_store(p, row, o);
            continue;
        }
        const T* z = (const T*)p.z + row * p.ldz;
        const T* zr = KL ? (const T*)p.zr + row * p.ldr : nullptr;
        const uint8_t* mask = p.mask ? p.mask + row * p.ldm : nullptr;
        const int act = p.act[row];
        const float za = mask && !mask[act] ? -INFINITY : el_f32(z[act]);
        RowSum q = wide_join<KL>(wide_sum<T, KL>(z, zr, mask, 0, p.A), s_sum);
        if (threadIdx.x < 64) {
            Coef c;
            row_finish<KL, double>(p, q, row, za, nullptr, c, o);
            if (threadIdx.x == 0) {
                s_coef = c;
                row_store(p, row, o);
                if (p.rec) rec_add(p, rec, row, o);
            }
        }
        __syncthreads();
        if (g) {
            const Coef c = s_coef;
            if (c.zero) wide_zero<T>(g, 0, p.A);
            else wide_grad<T, KL>(p, c, act, z, zr, mask, g, 0, p.A);
        }
        __syncthreads();                 // s_sum and s_coef are read
    }
    if (threadIdx.x == 0 && p.rec) p.rec[blockIdx.x] = rec;
}

// Few rows: pieces of rows to partial sums, then pieces again with the row's sums joined.
template <typename T, int KL>
__global__ __launch_bounds__(WR_THREADS) void loss_parts_kernel(const LossParams p) {
    __shared__ RowSum s_sum[WR_WAVES];
    const int64_t row = blockIdx.y;
    if (row_dead(p, row)) return;
    const int first = blockIdx.x * p.chunk, end = min(first + p.chunk, p.A);
    const T* z = (const T*)p.z + row * p.ldz;
    const uint8_t* mask = p.mask ? p.mask + row * p.ldm : nullptr;
    const RowSum q = wide_join<KL>(wide_sum<T, KL>(z, KL ? (const T*)p.zr + row * p.ldr : nullptr, mask, first, end), s_sum);
    if (threadIdx.x != 0) return;
    // (the gradient may go where the logits are, so the next launch does not look the action's logit up)
    const int act = p.act[row];
    Part& part = p.part[row * p.splits + blockIdx.x];
    part.r = q;
    part.za = act >= first && act < end && (!mask || mask[act]) ? el_f32(z[act]) : -INFINITY;
}
template <typename T, int KL>
__global__ __launch_bounds__(WR_THREADS) void loss_split_kernel(const LossParams p) {
    __shared__ RowSum s_sum[WR_WAVES];
    __shared__ Coef s_coef;
    const int64_t row = blockIdx.y;
    const int first = blockIdx.x * p.chunk, end = min(first + p.chunk, p.A);
    T* g = p.g ? (T*)p.g + row * p.ldg : nullptr;
    RowOut o = {0, 0, 0, 0, 0};
    const bool lead = blockIdx.x == 0 && threadIdx.x == 0;
    if (row_dead(p, row)) {
        if (g) wide_zero<T>(g, first, end);
        if (lead) {
            row_store(p, row, o);
            if (p.rec) p.rec[row] = {0, 0, 0, 0};
        }
        return;
    }
    RowSum q = row_empty();
    for (int i = threadIdx.x; i < p.splits; i += WR_THREADS) q = row_join<KL>(q, p.part[row * p.splits + i].r);
    q = wide_join<KL>(row_shuffle<KL>(q, 64), s_sum);
    const T* z = (const T*)p.z + row * p.ldz;
    const uint8_t* mask = p.mask ? p.mask + row * p.ldm : nullptr;
    const int act = p.act[row];
    if (threadIdx.x < 64) {
        Coef c;
        row_finish<KL, double>(p, q, row, p.part[row * p.splits + act / p.chunk].za, nullptr, c, o);
        if (threadIdx.x == 0) s_coef = c;
        if (lead) {
            row_store(p, row, o);
            Record rec = {0, 0, 0, 0};
            rec_add(p, rec, row, o);
            if (p.rec) p.rec[row] = rec;
        }
    }
    if (!g) return;
    __syncthreads();
    const Coef c = s_coef;
    if (c.zero) wide_zero<T>(g, first, end);
    else wide_grad<T, KL>(p, c, act, z, KL ? (const T*)p.zr + row * p.ldr : nullptr, mask, g, first, end);
}

// the records of a pass, in their order
__global__ __launch_bounds__(1024) void loss_stats_kernel(const Record* rec, int n, float scale, float* out) {
    __shared__ Record s_rec[16];
    Record r = {0, 0, 0, 0};
    for (int i = threadIdx.x; i < n; i += 1024) { r.loss += rec[i].loss; r.kl += rec[i].kl; r.ent += rec[i].ent; r.clipped += rec[i].clipped; }
    for (int k = 32; k > 0; k >>= 1) {
        r.loss += __shfl_xor(r.loss, k); r.kl += __shfl_xor(r.kl, k); r.ent += __shfl_xor(r.ent, k); r.clipped += __shfl_xor(r.clipped, k);
    }
    if ((threadIdx.x & 63) == 0) s_rec[threadIdx.x >> 6] = r;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int k = 1; k < 16; ++k) { r.loss += s_rec[k].loss; r.kl += s_rec[k].kl; r.ent += s_rec[k].ent; r.clipped += s_rec[k].clipped; }
        out[0] = (float)(scale * r.loss); out[1] = (float)(scale * r.kl); out[2] = (float)(scale * r.ent); out[3] = (float)(scale * r.clipped);
    }
}

int pl_fail(int code, const char* who, const char* what) {
    char msg[200];
    snprintf(msg, sizeof msg, "%s: %s", who, what);
    return set_error(code, msg);
}
int pl_launched(const char* who) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? ACCERL_OK : pl_fail(ACCERL_EHIP, who, hipGetErrorString(e));
}

template <typename T, int KL, int E>
void narrow_go(const LossParams& p, int G, int blocks, hipStream_t s) { loss_narrow_kernel<T, KL, E><<<dim3(blocks), dim3(NR_THREADS), 0, s>>>(p, G); }

template <typename T, int KL>
int loss_as(const char* who, LossParams& p, float* out_stats, hipStream_t s) {
    constexpr int VEC = 16 / sizeof(T);
    int records;
    if (p.A <= 512) {
        int G = 4;
        while (G * 8 < p.A) G *= 2;
        const int64_t want = (p.B + NR_THREADS / G - 1) / (NR_THREADS / G);
        records = (int)(want < PL_RECORDS ? want : PL_RECORDS);
        const int E = (p.A + G - 1) / G;
        if (E <= 2) narrow_go<T, KL, 2>(p, G, records, s);
        else if (E <= 4) narrow_go<T, KL, 4>(p, G, records, s);
        else if (E <= 6) narrow_go<T, KL, 6>(p, G, records, s);
        else narrow_go<T, KL, 8>(p, G, records, s);
    } else {
        // a row is split while there are fewer than 512 rows, into pieces of at least one vector a thread
        const int64_t pieces = (p.A + VEC * WR_THREADS - 1) / (VEC * WR_THREADS);
        int64_t splits = p.B < 512 ? 1024 / p.B : 1;
        if (splits > pieces) splits = pieces;
        p.chunk = (int)((pieces + splits - 1) / splits * VEC * WR_THREADS);
        p.splits = (p.A + p.chunk - 1) / p.chunk;
        if (p.splits > 1) {
            records = (int)p.B;
            loss_parts_kernel<T, KL><<<dim3(p.splits, (unsigned)p.B), dim3(WR_THREADS), 0, s>>>(p);
            if (int rc = pl_launched(who)) return rc;
            loss_split_kernel<T, KL><<<dim3(p.g ? p.splits : 1, (unsigned)p.B), dim3(WR_THREADS), 0, s>>>(p);
        } else {
            records = (int)(p.B < PL_RECORDS ? p.B : PL_RECORDS);
            loss_wide_kernel<T, KL><<<dim3(records), dim3(WR_THREADS), 0, s>>>(p);
        }
    }
    if (int rc = pl_launched(who)) return rc;
    if (!out_stats) return ACCERL_OK;
    loss_stats_kernel<<<dim3(1), dim3(1024), 0, s>>>(p.rec, records, p.scale, out_stats);
    return pl_launched(who);
}
template <typename T>
int loss_kl(const char* who, LossParams& p, float* out_stats, hipStream_t s) {
    if (p.kind == ACCERL_KL_FORWARD) return loss_as<T, 1>(who, p, out_stats, s);
    return p.kind == ACCERL_KL_REVERSE ? loss_as<T, 2>(who, p, out_stats, s) : loss_as<T, 0>(who, p, out_stats, s);
}
int loss_run(const char* who, int dtype, LossParams& p, float* out_stats, hipStream_t s) {
    if (dtype == ACCERL_DT_F32) return loss_kl<float>(who, p, out_stats, s);
    return dtype == ACCERL_DT_BF16 ? loss_kl<BF16>(who, p, out_stats, s) : loss_kl<F16>(who, p, out_stats, s);
}

constexpr int64_t PL_WORKSPACE = PL_RECORDS * (int64_t)sizeof(Record) + PL_PARTS * (int64_t)sizeof(Part);
bool pl_aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

// what every call checks; `done` is set where nothing is to be done
int check_table(const char* who, int32_t dtype, int64_t B, int64_t A, const void* z, int64_t ldz, const uint8_t* mask, int64_t ldm, const int32_t* act,
                const void* workspace, int64_t workspace_bytes, bool* done) {
    *done = false;
    if (!dtype_known(dtype)) return pl_fail(ACCERL_EINVAL, who, "unknown type of logits");
    if (B < 0 || A < 1) return pl_fail(ACCERL_EINVAL, who, "need B >= 0 and A >= 1");
    if (ldz < A) return pl_fail(ACCERL_EINVAL, who, "rows of logits overlap (stride < A)");
    if (mask && ldm != 0 && ldm < A) return pl_fail(ACCERL_EINVAL, who, "rows of the mask overlap (stride < A, and not 0)");
    if (A > PL_MAX_A || B > ((int64_t)1 << 31)) return pl_fail(ACCERL_EUNSUPPORTED, who, "more than 2^20 actions or 2^31 rows");
    if (B == 0) { *done = true; return ACCERL_OK; }
    if (!z || !act || !workspace) return pl_fail(ACCERL_EINVAL, who, "NULL argument");
    if (!pl_aligned(z, dtype_bytes(dtype)) || !pl_aligned(act, 4) || !pl_aligned(workspace, 16)) return pl_fail(ACCERL_EINVAL, who, "misaligned argument");
    if (workspace_bytes < PL_WORKSPACE) return pl_fail(ACCERL_EINVAL, who, "workspace smaller than accerl_policy_loss_workspace says");
    return ACCERL_OK;
}
void table_params(LossParams& p, int64_t B, int64_t A, const void* z, int64_t ldz, const uint8_t* mask, int64_t ldm, const int32_t* act, void* workspace) {
    p.B = B; p.A = (int)A; p.z = z; p.ldz = ldz; p.mask = mask; p.ldm = ldm; p.act = act;
    p.rec = (Record*)workspace;
    p.part = (Part*)((char*)workspace + PL_RECORDS * sizeof(Record));
}
bool overlap(const void* a, int64_t na, const void* b, int64_t nb) {
    return (uintptr_t)a < (uintptr_t)b + nb && (uintptr_t)b < (uintptr_t)a + na;
}
}  // namespace
}  // namespace accerl

using namespace accerl;

extern "C" {

int64_t accerl_policy_loss_workspace(void) { return PL_WORKSPACE; }

int accerl_action_logprob(const void* logits, int32_t dtype, int64_t ld_logits, const uint8_t* mask, int64_t ld_mask, const int32_t* actions,
                          int64_t B, int64_t A, float* out_logp, float* out_entropy, void* workspace, int64_t workspace_bytes, void* stream) {
    const char* who = "action_logprob";
    bool done;
    if (int rc = check_table(who, dtype, B, A, logits, ld_logits, mask, ld_mask, actions, workspace, workspace_bytes, &done)) return rc;
    if (done) return ACCERL_OK;
    if (!out_logp) return pl_fail(ACCERL_EINVAL, who, "NULL argument");
    if (!pl_aligned(out_logp, 4) || !pl_aligned(out_entropy, 4)) return pl_fail(ACCERL_EINVAL, who, "misaligned argument");
    LossParams p{};
    table_params(p, B, A, logits, ld_logits, mask, ld_mask, actions, workspace);
    p.rec = nullptr;
    p.only_lp = 1;
    p.lp = out_logp; p.ent = out_entropy;
    return loss_run(who, dtype, p, nullptr, (hipStream_t)stream);
}

int accerl_policy_loss(const accerl_policy_loss_args* a, void* stream) {
    const char* who = "policy_loss";
    if (!a) return pl_fail(ACCERL_EINVAL, who, "NULL argument");
    bool done;
    if (int rc = check_table(who, a->dtype, a->B, a->A, a->logits, a->ld_logits, a->mask, a->ld_mask, a->actions, a->workspace, a->workspace_bytes, &done)) return rc;
    if (a->kl_kind < ACCERL_KL_NONE || a->kl_kind > ACCERL_KL_REVERSE) return pl_fail(ACCERL_EINVAL, who, "unknown kind of KL term");
    const bool ref = a->kl_kind == ACCERL_KL_FORWARD || a->kl_kind == ACCERL_KL_REVERSE;
    if (!(a->clip_low >= 0.0) || !(a->clip_low <= 1.0) || !(a->clip_high >= 0.0)) return pl_fail(ACCERL_EINVAL, who, "need 0 <= clip_low <= 1 and clip_high >= 0");
    if (a->grad_logits && a->ld_grad < a->A) return pl_fail(ACCERL_EINVAL, who, "rows of the gradient overlap (stride < A)");
    if (ref && a->ld_ref < a->A) return pl_fail(ACCERL_EINVAL, who, "rows of the reference's logits overlap (stride < A)");
    if (done) return ACCERL_OK;
    if (!a->old_logp || !a->advantages || (ref && !a->ref_logits) || (a->kl_kind == ACCERL_KL_SAMPLED && !a->ref_logp))
        return pl_fail(ACCERL_EINVAL, who, "NULL input");
    const uintptr_t es = dtype_bytes(a->dtype);
    if (!pl_aligned(a->old_logp, 4) || !pl_aligned(a->advantages, 4) || !pl_aligned(a->weights, 4) || !pl_aligned(a->ref_logp, 4) ||
        !pl_aligned(a->out_loss, 4) || !pl_aligned(a->out_logp, 4) || !pl_aligned(a->out_kl, 4) || !pl_aligned(a->out_entropy, 4) ||
        !pl_aligned(a->out_stats, 4) || !pl_aligned(a->grad_logits, es) || (ref && !pl_aligned(a->ref_logits, es)))
        return pl_fail(ACCERL_EINVAL, who, "misaligned argument");
    if (a->grad_logits) {
        const int64_t n = ((a->B - 1) * a->ld_grad + a->A) * (int64_t)es, nz = ((a->B - 1) * a->ld_logits + a->A) * (int64_t)es;
        const bool in_place = a->grad_logits == a->logits && a->ld_grad == a->ld_logits;
        if (!in_place && overlap(a->grad_logits, n, a->logits, nz)) return pl_fail(ACCERL_EINVAL, who, "the gradient overlaps the logits and is not the same table");
        if (ref && overlap(a->grad_logits, n, a->ref_logits, ((a->B - 1) * a->ld_ref + a->A) * (int64_t)es))
            return pl_fail(ACCERL_EINVAL, who, "the gradient overlaps the reference's logits");
    }
    LossParams p{};
    table_params(p, a->B, a->A, a->logits, a->ld_logits, a->mask, a->ld_mask, a->actions, a->workspace);
    p.zr = ref ? a->ref_logits : nullptr; p.ldr = a->ld_ref;
    p.g = a->grad_logits; p.ldg = a->ld_grad;
    p.old = a->old_logp; p.adv = a->advantages; p.w = a->weights; p.ref_lp = a->ref_logp;
    p.loss = a->out_loss; p.lp = a->out_logp; p.kl = a->out_kl; p.ent = a->out_entropy;
    p.kind = a->kl_kind;
    p.lo = 1.0 - a->clip_low; p.hi = 1.0 + a->clip_high;
    p.ck = (float)a->kl_coef; p.ch = (float)a->entropy_coef; p.scale = (float)a->scale;
    if (!a->out_stats) p.rec = nullptr;
    return loss_run(who, a->dtype, p, a->out_stats, (hipStream_t)stream);
}

}  // extern "C"
