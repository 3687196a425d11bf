// Clipped policy loss with a KL term and an entropy term over wide action sets, its gradient, and the log-probabilities of actions.
// With z the logits of a row, z' the reference policy's, p = softmax(z), l = logsumexp(z), a the action:
//   lp = z_a - l,  r = exp(lp - old),  L = -min(r A, clip(r, 1 - lo, 1 + hi) A) + ck KL - ch H,  H = -sum p log p,
//   KL = sum p' log(p' / p) | sum p log(p / p') | exp(lr - lp) - (lr - lp) - 1.
// With m = max z, t_j = (z_j - m) log2 e, e_j = 2^t_j, s = sum e the gradient has one form for all kinds, with coefficients that are the row's:
//   dL/dz_j = e_j (c0 + c1 t_j + c2 (z_j - z'_j)) - c3 e'_j + ca [j = a].
// One pass over a row gives the maxima and the sums of e, e t, e' and e' (z' - z) or e (z - z'); the gradient is a second one, from registers
// as far as they hold the row.
#include <float.h>
#include <stdio.h>

#include <type_traits>

#include "wide_ops.h"

namespace accerl {
namespace {

constexpr int64_t PL_MAX_A = 1 << 20;
constexpr int PL_RECORDS = 2048;          // workgroups of a row pass, each leaves one record of sums
constexpr int PL_PARTS = 2048;            // pieces of rows, where a row is split
constexpr int PL_SPLIT = 256;             // rows below which one may be
// Vectors of a row that a lane of a wavefront holds at most; longer rows are a workgroup's (a workgroup each / a wavefront each, us: 10000 x 3000
// bf16 forward 104 / 78, 10000 x 2000 fp32 reverse 84.5 / 70.5, log-probabilities of 32827 x 1305 fp32 140 / 80).
constexpr int PL_HELD = 8;
constexpr int PL_SCALAR = 32;             // up to this many actions lanes take single elements
constexpr float PL_LOG2E = 1.44269504088896340736f;
constexpr double PL_LN2 = 0.693147180559945309417;

// the sums of a row or of a part of one under its maxima m and m'
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
    double* exact;           // split rows whose gradient goes where the logits are: a row's sum in 64 bits, or 0 where it is not next to a border
    int64_t B, ldz, ldr, ldg, ldm;
    int A, kind;             // accerl_kl_kind
    int only_lp;             // log-probabilities and entropies only
    int splits, chunk;       // pieces of a row, elements of a piece
    double lo, hi;           // the clipping borders themselves
    float log_lo, log_hi;    // their logarithms
    float ck, ch, scale;
    float* stats;            // out_stats where one workgroup does the pass (rec is then only a flag)
};

// A power is one multiply-add, t = z log2 e - c with c = m log2 e rounded once (what follows goes by that c), where the maximum lies within
// -50000 .. 2^20; for others the difference comes first, so that logits of any size lose nothing.
// A row is tried PLAIN first: all of its logits finite and both maxima in that range; masked places are at -59904, whose power is then 0,
// and no sum needs care for 0 * inf: 12 operations and two exponentials an element with a reference, where the careful form takes 19.  What
// is not like that gives sums that are no numbers, or a maximum out of that range, and is done again carefully: masked places at
// -inf, and a logit counts only where its probability is not 0.
constexpr float PL_LOW = -50000.0f, PL_HIGH = 0x1p20f;

struct Base { float c; bool far; };
__device__ __forceinline__ bool far_off(float m) { return !(m > PL_LOW && m < PL_HIGH); }

// what a row's gradient needs
struct Coef { Base z, r; float c0, c1, c2, c3, ca; int zero, plain; };

__device__ __forceinline__ float pl_exp2(float t) { return __builtin_amdgcn_exp2f(t); }     // results below 2^-126 may be 0
__device__ __forceinline__ RowSum row_empty() { return {-FLT_MAX, 0.0f, 0.0f, -FLT_MAX, 0.0f, 0.0f}; }
template <bool PLAIN> __device__ __forceinline__ Base base(float m) {
    const bool far = !PLAIN && far_off(m);
    return {far ? m : m * PL_LOG2E, far};
}
template <bool PLAIN> __device__ __forceinline__ float power(const Base& b, float z) {
    const float t = fmaf(z, PL_LOG2E, -b.c);
    return PLAIN || !b.far ? t : (z - b.c) * PL_LOG2E;
}

// Sums under a larger maximum.  The difference of maxima is kept finite so that an empty side's zeros stay zeros.
template <bool PLAIN> __device__ __forceinline__ float moved(float from, float to) {
    return fmaxf(PLAIN || !(far_off(from) || far_off(to)) ? from * PL_LOG2E - to * PL_LOG2E : (from - to) * PL_LOG2E, -FLT_MAX);
}
template <int KL, bool PLAIN>
__device__ __forceinline__ void row_raise(RowSum& a, float m, float mr) {
    const float d = moved<PLAIN>(a.m, m), f = pl_exp2(d);
    a.u = f * (a.u + a.s * d);
    a.s *= f;
    if constexpr (KL == 2) a.t *= f;
    a.m = m;
    if constexpr (KL != 0) {
        const float fr = pl_exp2(moved<PLAIN>(a.mr, mr));
        a.sr *= fr;
        if constexpr (KL == 1) a.t *= fr;
        a.mr = mr;
    }
}
template <int KL, bool PLAIN>
__device__ __forceinline__ RowSum row_join(RowSum a, RowSum b) {
    const float m = fmaxf(a.m, b.m), mr = fmaxf(a.mr, b.mr);
    row_raise<KL, PLAIN>(a, m, mr);
    row_raise<KL, PLAIN>(b, m, mr);
    a.s += b.s; a.u += b.u; a.sr += b.sr; a.t += b.t;
    return a;
}
// the sums take one element; c and cr are the bases of a's maxima
template <int KL, bool PLAIN>
__device__ __forceinline__ void row_add(RowSum& a, const Base& c, const Base& cr, float z, float zr) {
    const float t = power<PLAIN>(c, z), e = pl_exp2(t);
    a.s += e;
    a.u = fmaf(e, PLAIN ? t : fmaxf(t, -1500.0f), a.u);
    if constexpr (KL != 0) {
        const float er = pl_exp2(power<PLAIN>(cr, zr));
        a.sr += er;
        if constexpr (KL == 1) a.t = fmaf(er, PLAIN || er > 0.0f ? zr - z : 0.0f, a.t);
        else a.t = fmaf(e, PLAIN || e > 0.0f ? z - zr : 0.0f, a.t);
    }
}
// whether a plain row's joined sums hold
template <int KL, typename S>
__device__ __forceinline__ bool row_held(const S& a) {
    const bool z = !far_off(a.m) && fabs(a.s) < 1e30f && fabs(a.u) < 1e30f;
    return z && (KL == 0 || (!far_off(a.mr) && fabs(a.sr) < 1e30f && fabs(a.t) < 1e30f));
}
// the sums of neighbouring lanes joined, in all of them: under the common maxima first, so that a lane's sums are corrected once
template <int KL, bool PLAIN>
__device__ __forceinline__ RowSum row_shuffle(RowSum a, int lanes) {
    float m = a.m, mr = a.mr;
    for (int o = lanes >> 1; o > 0; o >>= 1) {
        m = fmaxf(m, __shfl_xor(m, o));
        if constexpr (KL != 0) mr = fmaxf(mr, __shfl_xor(mr, o));
    }
    row_raise<KL, PLAIN>(a, m, mr);
    for (int o = lanes >> 1; o > 0; o >>= 1) {
        a.s += __shfl_xor(a.s, o);
        a.u += __shfl_xor(a.u, o);
        if constexpr (KL != 0) { a.sr += __shfl_xor(a.sr, o); a.t += __shfl_xor(a.t, o); }
    }
    return a;
}

// the gradient at one element
template <int KL, bool PLAIN>
__device__ __forceinline__ float grad_at(const Coef& c, float z, float zr) {
    const float t = power<PLAIN>(c.z, z), e = pl_exp2(t);
    float k = fmaf(c.c1, PLAIN ? t : fmaxf(t, -1500.0f), c.c0);
    if constexpr (KL == 2) k = fmaf(c.c2, PLAIN ? z - zr : e == 0.0f ? 0.0f : fminf(z - zr, FLT_MAX), k);
    k *= e;
    if constexpr (KL == 1) k = fmaf(-c.c3, pl_exp2(power<PLAIN>(c.r, zr)), k);
    return k;
}

struct RowOut { float loss, lp, kl, ent, clipped; };
// a row's own numbers, asked for before its logits
struct RowIn { int act; float w, adv, old, ref_lp; };
__device__ __forceinline__ RowIn row_in(const LossParams& p, int64_t row) {
    RowIn r = {p.act[row], 1.0f, 0.0f, 0.0f, 0.0f};
    if (p.only_lp) return r;
    if (p.w) r.w = p.w[row];
    r.adv = p.adv[row];
    r.old = p.old[row];
    if (p.ref_lp) r.ref_lp = p.ref_lp[row];
    return r;
}
__device__ __forceinline__ bool row_dead(const LossParams& p, const RowIn& r) { return r.act < 0 || r.act >= p.A || r.w == 0.0f; }
// Next to a clipping border the side decides over a row's whole gradient: there the ratio is worked out in 64 bits.  "Next" is what 32 bits may
// be off by, which is relative for the ratio and absolute for its logarithm.  In half steps of 32 bits: `terms` for the sum (two or three dozen for its
// powers and joins, and one for each term that a lane adds up, all of which may be rounded the same way), `steps` of |log pi(a)| for its own roundings.
__device__ __forceinline__ bool near_border(const LossParams& p, float lp, float old, float terms, float steps) {
    const float r = lp - old, by = 0x1p-24f * fmaf(steps, fabsf(lp), terms);
    return fabsf(r - p.log_hi) < by || fabsf(r - p.log_lo) < by;
}
// A row's sums on their way to its scalars, in R.  kl: the KL where it was worked out more exactly (see loss_rows_kernel), negative: not known.
template <typename R> struct Sums { float m, mr; R s, u, sr, t, kl; };

__device__ __forceinline__ float pl_log2(float x) { return __builtin_amdgcn_logf(x); }      // of sums from 1 up and their quotients; 0 gives -inf
__device__ __forceinline__ double pl_log2(double x) { return log2(x); }
__device__ __forceinline__ float pl_exp(float x) { return expf(x); }
__device__ __forceinline__ double pl_exp(double x) { return exp(x); }
__device__ __forceinline__ float pl_inverse(float x) { return __builtin_amdgcn_rcpf(x); }    // to one unit in the last place
__device__ __forceinline__ double pl_inverse(double x) { return 1.0 / x; }

// exp(d) - d - 1, exact to its own size (in 32 bits the difference would leave a small one few digits): a series to d^8 below 1/2
__device__ __forceinline__ float exp_rest(float d) {
    if (fabsf(d) < 0.5f)
        return d * d * fmaf(d, fmaf(d, fmaf(d, fmaf(d, fmaf(d, fmaf(d, 1.0f / 40320, 1.0f / 5040), 1.0f / 720), 1.0f / 120), 1.0f / 24), 1.0f / 6), 0.5f);
    return d == INFINITY ? d : expf(d) - d - 1.0f;
}
__device__ __forceinline__ double exp_rest(double d) { return d == INFINITY ? d : exp(d) - d - 1.0; }
// its slope, exp(d) - 1: from 1/2 on not from the value, whose d takes the 1's digits (at -1e8 all of them) and whose -inf leaves no number
template <typename R> __device__ __forceinline__ R exp_slope(R d, R rest) { return fabs(d) < (R)0.5 ? rest + d : pl_exp(d) - (R)1; }
// log pi(a) in 64 bits from a row's 32-bit sum: what is subtracted from a reference's log-probability must not be rounded where that is.
// A function that is called, for its registers.
__device__ __attribute__((noinline)) double exact_logp(float za, float c, bool far, float s) {
    return PL_LN2 * ((far ? ((double)za - c) / PL_LN2 : (double)za * PL_LOG2E - c) - log2((double)s));
}

// Scalars of a row from its sums.  R: float where a wavefront holds many rows, double where the row is long and a wavefront does it once.
// The ratio may be replaced (`ratio`, a double) by one that was worked out more exactly.
template <int KL, typename R>
__device__ __forceinline__ void row_finish(const LossParams& p, const Sums<R>& q, bool plain, const RowIn& in, float za, const double* ratio, Coef& c, RowOut& o) {
    const bool empty = q.s == (R)0;
    const R ln2 = (R)PL_LN2, l2 = pl_log2(q.s), inv = pl_inverse(q.s);
    c.z = base<false>(q.m); c.r = base<false>(q.mr); c.plain = plain;
    // the power of the action, as the sum's terms have theirs
    const R ta = __is_same(R, float) ? (R)power<false>(c.z, za) : c.z.far ? ((R)za - (R)c.z.c) / ln2 : (R)za * (R)PL_LOG2E - (R)c.z.c;
    R lp = ln2 * (ta - l2);
    const R ent = ln2 * (l2 - q.u * inv);
    c.zero = empty;
    o.lp = empty ? -INFINITY : (float)lp;
    o.ent = empty ? 0.0f : (float)ent;
    o.loss = o.kl = o.clipped = 0.0f;
    if (p.only_lp) return;
    const float w = in.w, adv = in.adv;
    R away = (R)in.ref_lp - lp;
    if constexpr (__is_same(R, float) && KL == 0) {
        if (p.kind == ACCERL_KL_SAMPLED && !empty) {
            const double l = exact_logp(za, c.z.c, c.z.far, q.s);
            lp = (float)l;
            o.lp = lp;
            away = (float)(in.ref_lp - l);
        }
    }
    const R r = ratio ? (R)*ratio : lp == (R)-INFINITY ? (R)0 : pl_exp(lp - (R)in.old);
    const bool above = ratio ? *ratio > p.hi : r > (R)p.hi, below = ratio ? *ratio < p.lo : r < (R)p.lo;
    const bool cut = adv >= 0.0f ? above : below;
    const R pg = cut ? -(adv >= 0.0f ? (R)p.hi : (R)p.lo) * (R)adv : -r * (R)adv;
    R at = cut ? (R)0 : -r * (R)adv, kl = 0, c0 = 0, c2 = 0, c3 = 0;
    const R ck = p.ck, ch = p.ch;
    if constexpr (KL == 0) {
        if (p.kind == ACCERL_KL_SAMPLED) {
            kl = exp_rest(away);
            if (ck != (R)0) at -= ck * exp_slope(away, kl);
        }
    } else {
        const bool none = q.sr == (R)0;
        const R inv_r = pl_inverse(q.sr);
        const bool far = c.z.far || c.r.far;                      // l - l'
        const R dl = (far ? (R)q.m - (R)q.mr : ((R)c.z.c - (R)c.r.c) * ln2) + ln2 * pl_log2(q.s * inv_r);
        if constexpr (KL == 1) {
            if (!none) { kl = q.t * inv_r + dl; c0 = ck; c3 = ck * inv_r; }
        } else {
            kl = none ? (R)INFINITY : q.t * inv - dl;
        }
        if (q.kl >= (R)0 && kl < (R)0.5) kl = q.kl;
        if constexpr (KL == 2) {
            if (ck != (R)0) c0 = -ck * (dl + kl);
            c2 = ck;
        }
    }
    const R by = (R)w * (R)p.scale;
    c.c0 = (float)(by * inv * (c0 - at + ch * (ent - ln2 * l2)));
    c.c1 = (float)(by * inv * ch * ln2);
    c.c2 = (float)(by * inv * c2);
    c.c3 = (float)(by * c3);
    c.ca = (float)(by * at);
    if (empty) { o.ent = 0.0f; return; }
    o.kl = (float)kl;
    o.loss = (float)(pg + (ck == (R)0 ? (R)0 : ck * kl) - ch * ent);
    o.clipped = above || below ? 1.0f : 0.0f;
}

__device__ __forceinline__ void row_store(const LossParams& p, int64_t row, const RowOut& o) {
    if (p.loss) p.loss[row] = o.loss;
    if (p.lp) p.lp[row] = o.lp;
    if (p.kl) p.kl[row] = o.kl;
    if (p.ent) p.ent[row] = o.ent;
}
__device__ __forceinline__ void rec_stats(const Record& r, float scale, float* out) {
    out[0] = (float)(scale * r.loss); out[1] = (float)(scale * r.kl); out[2] = (float)(scale * r.ent); out[3] = (float)(scale * r.clipped);
}
__device__ __forceinline__ void rec_add(Record& r, float weight, const RowOut& o) {
    const double w = weight;
    r.loss += w * o.loss; r.kl += w * o.kl; r.ent += w * o.ent; r.clipped += w * o.clipped;
}

// ---------------------------------------------------------------- vectors of a row
// VEC elements of a row as they lie in memory (16 bytes, or one element of a narrow row); what is masked out, or no part of the row, is -inf.
template <typename T, int VEC> struct Vec {
    u32x4 w;
    __device__ __forceinline__ float at(int e) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
        else { float a, b; el_pair<T>(w[e / 2], a, b); return e & 1 ? b : a; }
    }
};
template <typename T> struct Vec<T, 1> {
    float w;
    __device__ __forceinline__ float at(int) const { return w; }
};
// what stands in a masked place: -59904 of a plain row, else -inf
template <typename T, bool PLAIN> constexpr uint32_t nothing() {
    if (PLAIN) return __is_same(T, float) ? 0xc76a0000u : __is_same(T, BF16) ? 0xc76ac76au : 0xfb50fb50u;
    return __is_same(T, float) ? 0xff800000u : __is_same(T, BF16) ? 0xff80ff80u : 0xfc00fc00u;
}
template <bool PLAIN> constexpr float nothing_f() { return PLAIN ? -59904.0f : -INFINITY; }

// Between two passes over a lane's vectors: what the first made of them (floats, powers) is made again in the second and not kept, which took
// every register of a wavefront.
template <typename T, int VEC, int N> __device__ __forceinline__ void vec_again(Vec<T, VEC> (&v)[N]) {
    if constexpr (VEC > 1) {
#pragma unroll
        for (int i = 0; i < N; ++i) asm volatile("" : "+v"(v[i].w));
    }
}

// A vector that would pass the end is moved back to end there (a row has VEC elements at least); what vectors before it have counts as
// masked, and of one past the end that is everything.
template <int VEC> __device__ __forceinline__ int vec_at(int i, int end) { return VEC == 1 ? i : min(i, end - VEC); }

// The lane as the compiler cannot follow it: it would work out every vector's addresses and conditions before the loop over the rows and
// keep them in registers.
__device__ __forceinline__ int opaque(int i) { asm volatile("" : "+v"(i)); return i; }

// `part` of a vector's element e in its word
template <typename T> __device__ __forceinline__ uint32_t vec_part(int e) { return sizeof(T) == 4 ? 0xffffffffu : e & 1 ? 0xffff0000u : 0xffffu; }
template <bool PLAIN, typename T, int VEC>
__device__ __forceinline__ void vec_drop(Vec<T, VEC>& v, int e) {
    constexpr int PER = 4 / (int)sizeof(T);
    v.w[e / PER] = (v.w[e / PER] & ~vec_part<T>(e)) | (nothing<T, PLAIN>() & vec_part<T>(e));
}
// 16 bytes of any alignment of elements; ONCE: nobody reads them again, they pass the caches by
template <bool ONCE, typename T> __device__ __forceinline__ u32x4 load16(const T* from) {
    if constexpr (sizeof(T) == 4) return ONCE ? __builtin_nontemporal_load((const u32x4_at4*)from) : *(const u32x4_at4*)from;
    else return ONCE ? __builtin_nontemporal_load((const u32x4_at2*)from) : *(const u32x4_at2*)from;
}
// FULL: the vector ends before the end.
template <bool FULL, bool PLAIN, bool ONCE = false, typename T, int VEC>
__device__ __forceinline__ void vec_load(Vec<T, VEC>& v, const T* row, const uint8_t* mask, int i, int end) {
    static_assert(VEC > 1, "whole vectors");
    {
        const int at = FULL ? i : vec_at<VEC>(i, end);
        v.w = load16<ONCE>(row + at);
        if (mask) {
#pragma unroll
            for (int k = 0; k < VEC / 4; ++k) {
                typedef uint32_t u32_at1 __attribute__((aligned(1)));
                const uint32_t m = *(const u32_at1*)(mask + at + 4 * k);
#pragma unroll
                for (int e = 0; e < 4; ++e) if (!((m >> (8 * e)) & 0xffu)) vec_drop<PLAIN>(v, 4 * k + e);
            }
        }
        if (!FULL && at != i) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) if (at + e < i) vec_drop<PLAIN>(v, e);
        }
    }
}
// Results are not read again here: they pass the caches by (2048 x 150000 bf16 with the forward KL 538 -> 496 us, 16000 x 6003 fp16 152 -> 123,
// 100000 x 300 fp32 163 -> 128).
template <bool FULL, typename T, int VEC>
__device__ __forceinline__ void vec_store(T* row, int i, int end, const float (&v)[VEC]) {
    if constexpr (VEC == 1) {
        if (i < end) row[i] = f32_el<T>(v[0]);
    } else if (FULL || i + VEC <= end) {
        if constexpr (VEC == 4) {
            const u32x4 w = {__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
            __builtin_nontemporal_store(w, (u32x4_at4*)(row + i));
        } else {
            u32x4 w;
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = f32_pair<T>(v[2 * e], v[2 * e + 1]);
            __builtin_nontemporal_store(w, (u32x4_at2*)(row + i));
        }
    } else {
        const int at = vec_at<VEC>(i, end);
#pragma unroll
        for (int e = 0; e < VEC; ++e) if (at + e >= i) row[at + e] = f32_el<T>(v[e]);
    }
}
// Elements j, j + G, .. of a narrow row; bit i of `allowed`: the i-th is part of the row.
template <bool PLAIN, typename T, int H>
__device__ __forceinline__ void single_load(Vec<T, 1> (&v)[H], const T* row, uint32_t allowed, int j, int G) {
#pragma unroll
    for (int i = 0; i < H; ++i) v[i].w = (allowed >> i) & 1 ? el_f32(row[j + i * G]) : nothing_f<PLAIN>();
}
template <int H>
__device__ __forceinline__ uint32_t single_allowed(const uint8_t* mask, int j, int G, int end) {
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < H; ++i)
        if (j + i * G < end && (!mask || mask[j + i * G])) bits |= 1u << i;
    return bits;
}

// the gradient of a vector's elements, to memory
template <bool FULL, int KL, bool PLAIN, typename T, int VEC>
__device__ __forceinline__ void vec_grad(const Coef& c, int act, const Vec<T, VEC>& z, const Vec<T, VEC>& zr, T* g, int i, int end) {
    float v[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = grad_at<KL, PLAIN>(c, z.at(e), KL ? zr.at(e) : 0.0f);
    const int a = act - (FULL ? i : vec_at<VEC>(i, end));
    if ((unsigned)a < (unsigned)VEC) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[e] += a == e ? c.ca : 0.0f;
    }
    vec_store<FULL>(g, i, end, v);
}
template <typename T, int VEC>
__device__ __forceinline__ void zero_row(T* g, int first, int end, int lane, int lanes) {
    float v[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = 0.0f;
    for (int i = first + lane * VEC; i < end; i += lanes * VEC) vec_store<false>(g, i, end, v);
}

// log2 of a quotient, off by a unit in the last place of a 32-bit logarithm: of a quotient near 1 that is far below 32 bits' step at 1
__device__ __forceinline__ double log2_close(double x) {
    const float y = (float)x;
    return (double)__builtin_amdgcn_logf(y) + (x - y) / y * 1.44269504088896340736;
}
// The ratio in 64 bits, from memory, by the lanes of a row.  A function that is called: it is hardly ever, and its registers would be every
// row's.
template <typename T>
__device__ __attribute__((noinline)) double exact_ratio(const T* z, const uint8_t* mask, int A, int j, int G, int step, float m, float za, float old) {
    double s = 0.0;
    for (int i = j * step; i < A; i += G * step)
        for (int e = i; e < min(i + step, A); ++e)
            if (!mask || mask[e]) s += exp((double)el_f32(z[e]) - (double)m);
    for (int k = G >> 1; k > 0; k >>= 1) s += __shfl_xor(s, k);
    return exp((double)za - (double)m - log(s) - (double)old);
}

// ---------------------------------------------------------------- rows that lanes of one wavefront hold
// G lanes hold a row, lane j its vectors j, j + G, ..  (H of them at most), read once.  A wavefront does 64 / G rows at a time.  Long batches
// of short rows are bound by instructions and the latency of a row's chain of sums, logarithm and gradient more than by memory: 262144 x 18
// fp32 with the forward KL and masks 35 us, of 14 that their bytes take at a copy's rate (a row a lane, through LDS, was
// faster from 9 to 18 actions by up to a sixth, and slower elsewhere by as much); 32 x 18 5.4 us in one launch, of which 4 is any launch that
// waits for memory.
constexpr int NR_THREADS = 256;
template <typename T, int KL, int VEC, int H>
__global__ __launch_bounds__(NR_THREADS) void loss_rows_kernel(const LossParams p, int G) {
    __shared__ Record s_rec[NR_THREADS / 64];
    const int tid = threadIdx.x;
    const int rows = NR_THREADS / G, shift = __builtin_ctz(G);
    Record rec = {0, 0, 0, 0};
    int64_t row = (int64_t)blockIdx.x * rows + tid / G;
    RowIn next = row_in(p, row < p.B ? row : p.B - 1);
    for (const int64_t stride = (int64_t)gridDim.x * rows; row < p.B; row += stride) {
        const int j = opaque(tid & (G - 1));
        const RowIn in = next;
        if (row + stride < p.B) next = row_in(p, row + stride);
        RowOut o = {0, 0, 0, 0, 0};
        T* g = p.g ? (T*)p.g + row * p.ldg : nullptr;
        if (row_dead(p, in)) {
            if (g) zero_row<T, VEC>(g, 0, p.A, j, G);
            if (j == 0) row_store(p, row, o);
            continue;
        }
        const T* z = (const T*)p.z + row * p.ldz;
        const T* zr = KL ? (const T*)p.zr + row * p.ldr : nullptr;
        const uint8_t* mask = p.mask ? p.mask + row * p.ldm : nullptr;
        const int act = in.act;
        Vec<T, VEC> a[H], b[H];
        RowSum q;
        float better_kl = -1.0f, za;
        uint32_t allowed = 0;                            // VEC == 1: this lane's elements; else whether the row has any, as far as the lane sees
        if constexpr (VEC == 1) allowed = single_allowed<H>(mask, j, G, p.A);
        else za = mask && !mask[act] ? -INFINITY : el_f32(z[act]);
        auto sums = [&](auto mode) {
            constexpr bool PLAIN = decltype(mode)::value;
            if constexpr (VEC == 1) {
                single_load<PLAIN>(a, z, allowed, j, G);
                if constexpr (KL != 0) single_load<PLAIN>(b, zr, allowed, j, G);
            } else {
#pragma unroll
                for (int i = 0; i < H; ++i) {
                    vec_load<false, PLAIN>(a[i], z, mask, (j + i * G) * VEC, p.A);
                    if constexpr (KL != 0) vec_load<false, PLAIN>(b[i], zr, mask, (j + i * G) * VEC, p.A);
                }
            }
            q = row_empty();
#pragma unroll
            for (int i = 0; i < H; ++i)
#pragma unroll
                for (int e = 0; e < VEC; ++e) { q.m = fmaxf(q.m, a[i].at(e)); if constexpr (KL != 0) q.mr = fmaxf(q.mr, b[i].at(e)); }
            for (int k = G >> 1; k > 0; k >>= 1) {
                q.m = fmaxf(q.m, __shfl_xor(q.m, k));
                if constexpr (KL != 0) q.mr = fmaxf(q.mr, __shfl_xor(q.mr, k));
            }
            const Base c = base<PLAIN>(q.m), cr = base<PLAIN>(q.mr);
            vec_again(a);
            if constexpr (KL != 0) vec_again(b);
#pragma unroll
            for (int i = 0; i < H; ++i) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) row_add<KL, PLAIN>(q, c, cr, a[i].at(e), KL ? b[i].at(e) : 0.0f);
                if (VEC > 1) __builtin_amdgcn_sched_barrier(0);      // (all vectors' elements at once would take every register)
            }
            // A small KL is the difference of sums that are hundreds of times larger, and 32-bit sums would leave it six digits.
            if constexpr (KL != 0 && VEC > 1) {
                // lanes' sums joined in 64 bits
                double ds = q.s, dsr = q.sr, dt = q.t;
                for (int k = G >> 1; k > 0; k >>= 1) { ds += __shfl_xor(ds, k); dsr += __shfl_xor(dsr, k); dt += __shfl_xor(dt, k); q.u += __shfl_xor(q.u, k); }
                q.s = (float)ds; q.sr = (float)dsr; q.t = (float)dt;
                const double apart = c.far || cr.far ? ((double)q.m - q.mr) / PL_LN2 : (double)c.c - cr.c;
                better_kl = (float)(KL == 1 ? dt / dsr + PL_LN2 * (apart + log2_close(ds / dsr)) : dt / ds - PL_LN2 * (apart + log2_close(ds / dsr)));
                better_kl = fmaxf(better_kl, 0.0f);
            } else {
                for (int k = G >> 1; k > 0; k >>= 1) {
                    q.s += __shfl_xor(q.s, k);
                    q.u += __shfl_xor(q.u, k);
                    if constexpr (KL != 0) { q.sr += __shfl_xor(q.sr, k); q.t += __shfl_xor(q.t, k); }
                }
            }
            if constexpr (KL != 0 && VEC == 1) {
                // With D_j the difference of logits less its mean under p' (forward) or p, KL = log E[exp(-D)] exactly, that is
                // log1p(E[exp(-D) - 1 + D]): a sum of small terms that are none of them negative.
                const float inv = pl_inverse(KL == 1 ? q.sr : q.s), mean = q.t * inv;
                float sum = 0.0f;
#pragma unroll
                for (int i = 0; i < H; ++i) {
                    const float x = a[i].at(0), y = b[i].at(0);
                    const float w = pl_exp2(KL == 1 ? power<PLAIN>(cr, y) : power<PLAIN>(c, x)), d = (KL == 1 ? y - x : x - y) - mean;
                    const float f = exp_rest(-d);
                    sum = fmaf(w, w > 0.0f ? f : 0.0f, sum);
                }
                for (int k = G >> 1; k > 0; k >>= 1) sum += __shfl_xor(sum, k);
                const float v = sum * inv, y = 1.0f + v;         // log(1 + v) = v log(y) / (y - 1), y as rounded
                better_kl = y == 1.0f ? v : (float)PL_LN2 * __builtin_amdgcn_logf(y) * v * __builtin_amdgcn_rcpf(y - 1.0f);
            }
        };
        sums(std::true_type());
        bool plain = row_held<KL>(q);
        if (!plain && mask && q.m == nothing_f<true>()) {
            // a row that the mask leaves empty, most likely: not to be done again
            uint32_t any = allowed;
            if constexpr (VEC > 1)
                for (int i = j; i < p.A; i += G) any |= mask[i];
            for (int k = G >> 1; k > 0; k >>= 1) any |= (uint32_t)__shfl_xor((int)any, k);
            if (!any) { q = row_empty(); plain = true; }
        }
        if (!plain) sums(std::false_type());             // (all lanes of a row alike)
        if constexpr (VEC == 1) {
            // the action's logit from the lane that holds it
            const int held = act >> shift;
            float v = a[0].w;
#pragma unroll
            for (int i = 1; i < H; ++i) v = held == i ? a[i].w : v;
            v = (allowed >> held) & 1 ? v : -INFINITY;
            za = __shfl(v, (tid & 63 & ~(G - 1)) | (act & (G - 1)));
        }
        Coef c;
        double ratio;
        const double* better = nullptr;
        if (!p.only_lp && q.s > 0.0f) {
            // (all lanes of a row branch alike)
            const float lp = (float)PL_LN2 * (power<false>(base<false>(q.m), za) - pl_log2(q.s));
            if (near_border(p, lp, in.old, 40.0f + H * VEC, 4.0f)) {
                ratio = exact_ratio<T>(z, mask, p.A, j, G, VEC, q.m, za, in.old);
                better = &ratio;
            }
        }
        const Sums<float> joined = {q.m, q.mr, q.s, q.u, q.sr, q.t, better_kl};
        row_finish<KL, float>(p, joined, plain, in, za, better, c, o);
        if (g) {
            if (c.zero) zero_row<T, VEC>(g, 0, p.A, j, G);
            else {
                auto grads = [&](auto mode) {
                    vec_again(a);
                    if constexpr (KL != 0) vec_again(b);
#pragma unroll
                    for (int i = 0; i < H; ++i) {
                        if ((j + i * G) * VEC < p.A) vec_grad<false, KL, decltype(mode)::value>(c, act, a[i], b[i], g, (j + i * G) * VEC, p.A);
                        if (VEC > 1) __builtin_amdgcn_sched_barrier(0);
                    }
                };
                if (plain) grads(std::true_type());
                else grads(std::false_type());
            }
        }
        if (j == 0) {
            row_store(p, row, o);
            if (p.rec) rec_add(rec, in.w, o);
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
        if (p.stats) rec_stats(rec, p.scale, p.stats);
        else p.rec[blockIdx.x] = rec;
    }
}

// ---------------------------------------------------------------- wide rows: a workgroup holds one, or a piece of one
constexpr int WR_THREADS = 256;
constexpr int WR_WAVES = 8;               // most wavefronts of a workgroup

// The vectors of elements first to end, U at a time, loaded together and ahead of the ones before; the last ones one by one.  f(whole,
// vectors, vectors of the reference, first element): `whole` (a type) where no vector passes the end.
template <typename T, int KL, int THREADS, int U, bool PLAIN, bool ONCE = false, typename F>
__device__ __forceinline__ void wide_stream(const T* z, const T* zr, const uint8_t* mask, int first, int end, F&& f) {
    constexpr int VEC = 16 / sizeof(T), STEP = THREADS * VEC;
    Vec<T, VEC> a[U], b[U];
    int i = first + opaque(threadIdx.x) * VEC;
    auto load = [&](auto whole, int at) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            vec_load<decltype(whole)::value, PLAIN, ONCE>(a[u], z, mask, at + u * STEP, end);
            if constexpr (KL != 0) vec_load<decltype(whole)::value, PLAIN, ONCE>(b[u], zr, mask, at + u * STEP, end);
        }
    };
    const int turns = (end - first) / (U * STEP);              // whole ones
    if (turns > 0) {
        load(std::true_type(), i);
        for (int k = 1; k <= turns; ++k, i += U * STEP) {
            Vec<T, VEC> x[U], y[U];
#pragma unroll
            for (int u = 0; u < U; ++u) { x[u] = a[u]; if constexpr (KL != 0) y[u] = b[u]; }
            if (k < turns) load(std::true_type(), i + U * STEP);
            f(std::true_type(), x, y, i);
        }
    }
    // the rest, as many vectors as there are (the whole workgroup alike)
    const int rest = first + turns * (U * STEP);
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (rest + u * STEP < end) {
            vec_load<false, PLAIN, ONCE>(a[u], z, mask, i + u * STEP, end);
            if constexpr (KL != 0) vec_load<false, PLAIN, ONCE>(b[u], zr, mask, i + u * STEP, end);
        }
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (rest + u * STEP < end) {
            const Vec<T, VEC> x[1] = {a[u]}, y[1] = {b[u]};
            f(std::false_type(), x, y, i + u * STEP);
        }
}
// vectors `first` to `first + N` of an array
template <int KL, int N, bool PLAIN, typename T, int VEC, int ALL>
__device__ __forceinline__ void sum_vecs(RowSum& q, const Vec<T, VEC> (&x)[ALL], const Vec<T, VEC> (&y)[ALL], int first) {
    float m = q.m, mr = q.mr;
#pragma unroll
    for (int u = 0; u < N; ++u)
#pragma unroll
        for (int e = 0; e < VEC; ++e) { m = fmaxf(m, x[first + u].at(e)); if constexpr (KL != 0) mr = fmaxf(mr, y[first + u].at(e)); }
    row_raise<KL, PLAIN>(q, m, mr);
    const Base c = base<PLAIN>(m), cr = base<PLAIN>(mr);
    // (among themselves first: a lane's sum is then rounded once for all of them)
    RowSum own = {m, 0.0f, 0.0f, mr, 0.0f, 0.0f};
#pragma unroll
    for (int u = 0; u < N; ++u)
#pragma unroll
        for (int e = 0; e < VEC; ++e) row_add<KL, PLAIN>(own, c, cr, x[first + u].at(e), KL ? y[first + u].at(e) : 0.0f);
    q.s += own.s; q.u += own.u;
    if constexpr (KL != 0) { q.sr += own.sr; q.t += own.t; }
}

// Terms of a lane's sum, as near_border counts them: those of up to four vectors among themselves, then two vectors a time, each time once more and three
// where the maximum rises.
template <int VEC> __device__ __forceinline__ float wide_terms(int elements, int threads) {
    return 24.0f + 4 * VEC + 4.0f * (2.0f + (float)elements / (float)(2 * VEC * threads));
}

// What the workgroup of a row shares.  The row's scalars are worked out by wavefront 0 in 64 bits, in a function that is called: inside the
// kernels its registers, and constants that the compiler keeps for the next row, would be everybody's.
struct WideShared {
    LossParams p;
    RowSum sum[WR_WAVES];
    Coef coef;
    RowOut out;
    Record rec;              // the sums of the workgroup's rows, thread 0's: in registers they would be everybody's
    int waves;
    float m;                 // the row's maximum
    double exact[WR_WAVES];
};
// EXACT: with the ratio that the sum in `exact` gives.
template <int KL, bool EXACT>
__device__ __attribute__((noinline)) void wide_finish(WideShared* w, bool plain, RowIn in, float za) {
    Sums<double> r = {-FLT_MAX, -FLT_MAX, 0.0, 0.0, 0.0, 0.0, -1.0};
    for (int k = 0; k < w->waves; ++k) { r.m = fmaxf(r.m, w->sum[k].m); r.mr = fmaxf(r.mr, w->sum[k].mr); }
    for (int k = 0; k < w->waves; ++k) {
        const RowSum s = w->sum[k];
        const double d = plain ? moved<true>(s.m, r.m) : moved<false>(s.m, r.m), f = pl_exp2((float)d);
        const double fr = KL ? pl_exp2(plain ? moved<true>(s.mr, r.mr) : moved<false>(s.mr, r.mr)) : 0.0;
        r.s += f * s.s;
        r.u += f * (s.u + s.s * d);
        r.sr += fr * s.sr;
        r.t += (KL == 2 ? f : fr) * s.t;
    }
    Coef c;
    RowOut o;
    double ratio = 0.0;
    if constexpr (EXACT) {
        for (int k = 0; k < w->waves; ++k) ratio += w->exact[k];
        ratio = exp((double)za - (double)r.m - log(ratio) - (double)in.old);
    }
    row_finish<KL, double>(w->p, r, plain, in, za, EXACT ? &ratio : nullptr, c, o);
    if (plain && !row_held<KL>(r)) c.plain = -1;                  // to be done again
    if (threadIdx.x == 0) { w->coef = c; w->out = o; w->m = r.m; }
}
// The row's sum in 64 bits, from memory, by the whole workgroup: the wavefronts' parts go to `w->exact`.  A function that is called, like the one
// above; four elements a lane are on their way while four are summed (one after the other a masked row of 50000 took 150 us, like this, its
// gradient read again, 38; eight take more registers than some of the kernels have).
template <int THREADS, typename T>
__device__ __attribute__((noinline)) void exact_sum(WideShared* w, const T* z, const uint8_t* mask) {
    const int A = w->p.A;
    const double m = w->m;
    double s = 0.0;
    float v[4], next[4];
    const auto load = [&](float (&d)[4], int i) {
#pragma unroll
        for (int k = 0; k < 4; ++k) d[k] = el_f32(z[min(i + k * THREADS, A - 1)]);
        if (mask) {
#pragma unroll
            for (int k = 0; k < 4; ++k) if (!mask[min(i + k * THREADS, A - 1)]) d[k] = -INFINITY;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) if (i + k * THREADS >= A) d[k] = -INFINITY;
    };
    load(v, threadIdx.x);
    for (int i = threadIdx.x; i < A; i += 4 * THREADS) {
        load(next, i + 4 * THREADS);
#pragma unroll
        for (int k = 0; k < 4; ++k) { s += exp((double)v[k] - m); v[k] = next[k]; }
    }
    for (int k = 32; k > 0; k >>= 1) s += __shfl_xor(s, k);
    if ((threadIdx.x & 63) == 0) w->exact[threadIdx.x >> 6] = s;
}
// The row's coefficients, to everybody, and its outputs, to thread 0 (`w.out`).
template <int KL, bool PLAIN>
__device__ __forceinline__ Coef wide_coef(WideShared& w, const RowSum& q, const RowIn& in, float za) {
    if ((threadIdx.x & 63) == 0) w.sum[threadIdx.x >> 6] = q;
    __syncthreads();
    if (threadIdx.x < 64) wide_finish<KL, false>(&w, PLAIN, in, za);
    __syncthreads();
    return w.coef;
}

// The vectors tid, THREADS + tid, .. of a row, whole ones.  All are requested before anything is done with one; a mask is seen to afterwards.
template <int THREADS, typename T, int VEC, int H>
__device__ __forceinline__ void held_load(Vec<T, VEC> (&v)[H], const T* row, int tid) {
#pragma unroll
    for (int i = 0; i < H; ++i) {
        // (past the caches: 8192 x 32000 bf16 222 -> 209 us, 12500 x 2 x 16000 295 -> 285, but with two of three vectors held 16000 x 6003 fp16
        // 123 -> 139)
        v[i].w = load16<(H >= 4)>((const T*)((const char*)row + (uint32_t)((i * THREADS + tid) * 16)));
    }
}
template <bool TWO, int THREADS, typename T, int VEC, int H>
__device__ __forceinline__ void held_mask(Vec<T, VEC> (&a)[H], Vec<T, VEC> (&b)[H], const uint8_t* mask, int tid) {
#pragma unroll
    for (int i = 0; i < H; ++i) {
#pragma unroll
        for (int k = 0; k < VEC / 4; ++k) {
            typedef uint32_t u32_at1 __attribute__((aligned(1)));
            const uint32_t m = *(const u32_at1*)(mask + (uint32_t)((i * THREADS + tid) * VEC + 4 * k));
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (!((m >> (8 * e)) & 0xffu)) { vec_drop<true>(a[i], 4 * k + e); if (TWO) vec_drop<true>(b[i], 4 * k + e); }
        }
        __builtin_amdgcn_sched_barrier(0);
    }
}

template <int KL, typename T, int VEC, int H>
__device__ __forceinline__ void held_sums(RowSum& q, const Vec<T, VEC> (&a)[H], const Vec<T, VEC> (&b)[H]) {
#pragma unroll
    for (int i = 0; i + 2 <= H; i += 2) {
        sum_vecs<KL, 2, true>(q, a, b, i);
        __builtin_amdgcn_sched_barrier(0);                          // (more of them at once would take more registers)
    }
    if constexpr (H % 2) sum_vecs<KL, 1, true>(q, a, b, H - 1);
}

// Rows one after the other, each by the whole workgroup.  H vectors of a row, all of them inside it, stay in a lane's registers from the sums
// to the gradient, and up to LDS more (of each table) in LDS, a lane's own; the rest is read twice.  Bound by memory, a row's two to three
// tables once where all of it is held: what misses the second-level cache moves at one rate whether the last-level cache has it or not, so
// that a second reading costs what the first did.  Four workgroups of 256 a compute unit hold 15 vectors (eight of each table: more registers
// would spill, and seven did), two hold 56 (28) and one of 512 112 (56): fewer wavefronts hide less, but what they save is more from rows of
// 15 to 30 vectors a lane on.  8192 x 32000 bf16, no reference: 206 us, 5.1 TB/s of once read and once written; 2048 x 2 x 150000 486, 3.8.
// LOSS: not log-probabilities alone, which have no gradient and no border to be next to, and need not have these' registers.
template <typename T, int KL, int H, int THREADS, int PER_SIMD, int LDS, bool LOSS>
__global__ __launch_bounds__(THREADS, PER_SIMD) void loss_wide_kernel(const LossParams p) {
    constexpr int VEC = 16 / sizeof(T), U = KL ? 2 : 4, HELD = H * THREADS * VEC;
    __shared__ WideShared w;
    __shared__ u32x4 s_row[LDS > 0 ? LDS * (KL ? 2 : 1) : 1][LDS > 0 ? THREADS : 1];     // vectors behind those in registers, a lane's own
    if (threadIdx.x == 0) { w.p = p; w.rec = {0, 0, 0, 0}; w.waves = THREADS / 64; }
    for (int64_t row = blockIdx.x; row < p.B; row += gridDim.x) {
        const int tid = opaque(threadIdx.x);
        T* g = LOSS && p.g ? (T*)p.g + row * p.ldg : nullptr;
        const RowIn in = row_in(p, row);
        if (row_dead(p, in)) {
            if (g) zero_row<T, VEC>(g, 0, p.A, tid, THREADS);
            if (tid == 0) row_store(p, row, {0, 0, 0, 0, 0});
            continue;
        }
        const T* z = (const T*)p.z + row * p.ldz;
        const T* zr = KL ? (const T*)p.zr + row * p.ldr : nullptr;
        const uint8_t* mask = p.mask ? p.mask + row * p.ldm : nullptr;
        const int act = in.act;
        const float za = mask && !mask[act] ? -INFINITY : el_f32(z[act]);
        Vec<T, VEC> a[H], b[H];
        held_load<THREADS>(a, z, tid);
        if constexpr (KL != 0) held_load<THREADS>(b, zr, tid);
        if (mask) held_mask<KL != 0, THREADS>(a, b, mask, opaque(tid));
        RowSum q = row_empty();
        held_sums<KL>(q, a, b);
        const auto take = [&](auto, const auto& x, const auto& y, int at) {
            constexpr int N = sizeof(x) / sizeof(x[0]);
            if constexpr (LDS > 0) {
                const int slot = (at - HELD) / (THREADS * VEC);
#pragma unroll
                for (int u = 0; u < N; ++u)
                    if (slot + u < LDS) {
                        s_row[slot + u][tid] = x[u].w;
                        if constexpr (KL != 0) s_row[LDS + slot + u][tid] = y[u].w;
                    }
            }
            sum_vecs<KL, N, true>(q, x, y, 0);
        };
        // (without a gradient nothing is read twice: log-probabilities of 4096 x 32768 fp32 105 -> 95 us)
        if (H <= 4 && !g) wide_stream<T, KL, THREADS, U, true, true>(z, zr, mask, HELD, p.A, take);
        else wide_stream<T, KL, THREADS, U, true>(z, zr, mask, HELD, p.A, take);
        Coef c = wide_coef<KL, true>(w, row_shuffle<KL, true>(q, 64), in, za);
        const auto put = [&] {
            if (tid == 0) {
                row_store(p, row, w.out);
                if (p.rec) rec_add(w.rec, in.w, w.out);
            }
        };
        const auto near = [&] { return LOSS && near_border(p, w.out.lp, in.old, wide_terms<VEC>(p.A, THREADS), 2.0f); };
        const auto exact = [&] {
            exact_sum<THREADS>(&w, z, mask);
            __syncthreads();
            if (threadIdx.x < 64) wide_finish<KL, true>(&w, c.plain, in, za);
            __syncthreads();
            c = w.coef;
        };
        const auto grads = [&](auto mode, auto n, int first) {
            constexpr int N = decltype(n)::value;
            constexpr bool PLAIN = decltype(mode)::value;
            wide_stream<T, KL, THREADS, N, PLAIN>(z, zr, mask, first, p.A, [&](auto full, const auto& x, const auto& y, int i) {
#pragma unroll
                for (int u = 0; u < (int)(sizeof(x) / sizeof(x[0])); ++u)
                    if (decltype(full)::value || i + u * THREADS * VEC < p.A)
                        vec_grad<decltype(full)::value, KL, PLAIN>(c, act, x[u], y[u], g, i + u * THREADS * VEC, p.A);
            });
        };
        if (c.plain < 0) {                                          // (everybody)
            q = row_empty();
            wide_stream<T, KL, THREADS, 1, false>(z, zr, mask, 0, p.A, [&](auto, const auto& x, const auto& y, int) { sum_vecs<KL, sizeof(x) / sizeof(x[0]), false>(q, x, y, 0); });
            q = row_shuffle<KL, false>(q, 64);
            __syncthreads();
            c = wide_coef<KL, false>(w, q, in, za);
            if (near()) exact();
            put();
            if (g) {
                if (c.zero) zero_row<T, VEC>(g, 0, p.A, tid, THREADS);
                else grads(std::false_type(), std::integral_constant<int, 1>(), 0);
            }
        } else {
            int first = 0;                                          // where the part of the row begins that is read again
            if (near()) {                                           // (everybody) all of it: what is held would take registers over the calls
                exact();
                put();
            } else {
                put();
                if (g) {
                    vec_again(a);
                    if constexpr (KL != 0) vec_again(b);
                    const int lane = opaque(tid);
#pragma unroll
                    for (int i = 0; i < H; ++i) {
                        vec_grad<true, KL, true>(c, act, a[i], b[i], g, (i * THREADS + lane) * VEC, p.A);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                    const int rest = (p.A - HELD) / (THREADS * VEC), kept = rest < LDS ? rest : LDS;      // whole vectors in LDS
                    if constexpr (LDS > 0) {
#pragma unroll 1
                        for (int i = 0; i < kept; ++i) {
                            Vec<T, VEC> x, y;
                            x.w = s_row[i][lane];
                            if constexpr (KL != 0) y.w = s_row[LDS + i][lane];
                            vec_grad<true, KL, true>(c, act, x, y, g, ((H + i) * THREADS + lane) * VEC, p.A);
                        }
                    }
                    first = HELD + kept * THREADS * VEC;
                }
            }
            if (g) grads(std::true_type(), std::integral_constant<int, U>(), first);
        }
        __syncthreads();                 // w.sum and w.coef are read
    }
    if (threadIdx.x == 0 && p.rec) p.rec[blockIdx.x] = w.rec;
}

// Few rows: pieces of rows to partial sums, then pieces again with the row's sums joined.  Two dependent launches, latency: 16 x 100000
// bf16 log-probabilities 4.8 + 6.0 us.  (One launch would need its workgroups to wait for each other or memory that is cleared between calls.)
constexpr int SP_THREADS = 512;
template <typename T, int KL>
__global__ __launch_bounds__(SP_THREADS) void loss_parts_kernel(const LossParams p) {
    constexpr int U = 2;
    __shared__ RowSum s_sum[WR_WAVES];
    const int64_t row = blockIdx.y;
    const RowIn in = row_in(p, row);
    if (row_dead(p, in)) return;
    const int first = blockIdx.x * p.chunk, end = min(first + p.chunk, p.A);
    const T* z = (const T*)p.z + row * p.ldz;
    const uint8_t* mask = p.mask ? p.mask + row * p.ldm : nullptr;
    RowSum q = row_empty();
    wide_stream<T, KL, SP_THREADS, U, false>(z, KL ? (const T*)p.zr + row * p.ldr : nullptr, mask, first, end,
                          [&](auto, const auto& x, const auto& y, int) { sum_vecs<KL, sizeof(x) / sizeof(x[0]), false>(q, x, y, 0); });
    q = row_shuffle<KL, false>(q, 64);
    if ((threadIdx.x & 63) == 0) s_sum[threadIdx.x >> 6] = q;
    __syncthreads();
    if (threadIdx.x >= 64) return;
    q = row_shuffle<KL, false>(s_sum[threadIdx.x & (WR_WAVES - 1)], WR_WAVES);
    if (threadIdx.x != 0) return;
    // (the gradient may go where the logits are, so the next launch does not look the action's logit up)
    const int act = in.act;
    Part& part = p.part[row * p.splits + blockIdx.x];
    part.r = q;
    part.za = act >= first && act < end && (!mask || mask[act]) ? el_f32(z[act]) : -INFINITY;
}
// whether a row of pieces is next to a border (three a level for the joins of pieces)
template <int VEC> __device__ __forceinline__ bool split_near(const LossParams& p, const WideShared& w, const RowIn& in) {
    return near_border(p, w.out.lp, in.old, 24.0f + wide_terms<VEC>(p.chunk, SP_THREADS), 2.0f);
}
// Between the two, where the gradient goes where the logits are: a row next to a border is summed in 64 bits before any of it is overwritten.
template <typename T>
__global__ __launch_bounds__(SP_THREADS) void loss_border_kernel(const LossParams p) {
    __shared__ WideShared w;
    const int64_t row = blockIdx.x;
    const RowIn in = row_in(p, row);
    if (row_dead(p, in)) return;
    if (threadIdx.x == 0) { w.p = p; w.waves = SP_THREADS / 64; }
    RowSum q = row_empty();
    for (int i = threadIdx.x; i < p.splits; i += SP_THREADS) q = row_join<0, false>(q, p.part[row * p.splits + i].r);
    wide_coef<0, false>(w, row_shuffle<0, false>(q, 64), in, p.part[row * p.splits + in.act / p.chunk].za);
    const bool near = split_near<16 / (int)sizeof(T)>(p, w, in);                         // (everybody)
    if (near) exact_sum<SP_THREADS>(&w, (const T*)p.z + row * p.ldz, p.mask ? p.mask + row * p.ldm : nullptr);
    __syncthreads();
    if (threadIdx.x != 0) return;
    double s = 0.0;
    if (near) for (int k = 0; k < w.waves; ++k) s += w.exact[k];
    p.exact[row] = s;
}
// LOSS: as above; what the border takes costs the 10 us of few rows' log-probabilities half a one.
template <typename T, int KL, bool LOSS>
__global__ __launch_bounds__(SP_THREADS) void loss_split_kernel(const LossParams p) {
    constexpr int VEC = 16 / sizeof(T), U = 2;
    __shared__ WideShared w;
    const int64_t row = blockIdx.y;
    const int first = blockIdx.x * p.chunk, end = min(first + p.chunk, p.A);
    T* g = p.g ? (T*)p.g + row * p.ldg : nullptr;
    const bool lead = blockIdx.x == 0 && threadIdx.x == 0;
    const RowIn in = row_in(p, row);
    if (row_dead(p, in)) {
        if (g) zero_row<T, VEC>(g, first, end, threadIdx.x, SP_THREADS);
        if (lead) {
            row_store(p, row, {0, 0, 0, 0, 0});
            if (p.rec) p.rec[row] = {0, 0, 0, 0};
        }
        return;
    }
    if (threadIdx.x == 0) { w.p = p; w.waves = SP_THREADS / 64; }
    RowSum q = row_empty();
    for (int i = threadIdx.x; i < p.splits; i += SP_THREADS) q = row_join<KL, false>(q, p.part[row * p.splits + i].r);
    const int act = in.act;
    const float za = p.part[row * p.splits + act / p.chunk].za;
    Coef c = wide_coef<KL, false>(w, row_shuffle<KL, false>(q, 64), in, za);
    const T* z = (const T*)p.z + row * p.ldz;
    const uint8_t* mask = p.mask ? p.mask + row * p.ldm : nullptr;
    if (LOSS && (p.exact ? p.exact[row] != 0.0 : split_near<VEC>(p, w, in))) {     // (everybody)
        if (!p.exact) exact_sum<SP_THREADS>(&w, z, mask);
        else if (threadIdx.x < SP_THREADS / 64) w.exact[threadIdx.x] = threadIdx.x == 0 ? p.exact[row] : 0.0;
        __syncthreads();
        if (threadIdx.x < 64) wide_finish<KL, true>(&w, false, in, za);
        __syncthreads();
        c = w.coef;
    }
    if (lead) {
        row_store(p, row, w.out);
        Record rec = {0, 0, 0, 0};
        rec_add(rec, in.w, w.out);
        if (p.rec) p.rec[row] = rec;
    }
    if (!g) return;
    if (c.zero) zero_row<T, VEC>(g, first, end, threadIdx.x, SP_THREADS);
    else
        wide_stream<T, KL, SP_THREADS, U, false>(z, KL ? (const T*)p.zr + row * p.ldr : nullptr, mask, first, end,
                              [&](auto full, const auto& x, const auto& y, int i) {
#pragma unroll
                                  for (int u = 0; u < (int)(sizeof(x) / sizeof(x[0])); ++u)
                                      if (decltype(full)::value || i + u * SP_THREADS * VEC < end)
                                          vec_grad<decltype(full)::value, KL, false>(c, act, x[u], y[u], g, i + u * SP_THREADS * VEC, end);
                              });
}

// the records of a pass, in their order, so that sums repeat: 2048 of them 5 us, a launch and two round trips
__global__ __launch_bounds__(1024) void loss_stats_kernel(const Record* rec, int n, float scale, float* out) {
    __shared__ Record s_rec[16];
    Record r = {0, 0, 0, 0};
    for (int i = threadIdx.x; i < n; i += (int)blockDim.x) { r.loss += rec[i].loss; r.kl += rec[i].kl; r.ent += rec[i].ent; r.clipped += rec[i].clipped; }
    for (int k = 32; k > 0; k >>= 1) {
        r.loss += __shfl_xor(r.loss, k); r.kl += __shfl_xor(r.kl, k); r.ent += __shfl_xor(r.ent, k); r.clipped += __shfl_xor(r.clipped, k);
    }
    if ((threadIdx.x & 63) == 0) s_rec[threadIdx.x >> 6] = r;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int k = 1; k < (int)blockDim.x / 64; ++k) { r.loss += s_rec[k].loss; r.kl += s_rec[k].kl; r.ent += s_rec[k].ent; r.clipped += s_rec[k].clipped; }
        rec_stats(r, scale, out);
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

template <typename T, int KL, int VEC, int H>
void rows_go(const LossParams& p, int G, int blocks, hipStream_t s) { loss_rows_kernel<T, KL, VEC, H><<<dim3(blocks), dim3(NR_THREADS), 0, s>>>(p, G); }

template <typename T, int KL, int H, int THREADS, int PER_SIMD, int LDS, bool LOSS = true>
void wide_go(const LossParams& p, int blocks, hipStream_t s) { loss_wide_kernel<T, KL, H, THREADS, PER_SIMD, LDS, LOSS><<<dim3(blocks), dim3(THREADS), 0, s>>>(p); }

template <typename T, int KL>
int loss_as(const char* who, LossParams& p, float* out_stats, hipStream_t s) {
    constexpr int VEC = 16 / sizeof(T);
    int records;
    if (p.A <= 64 * VEC * PL_HELD) {
        const int vec = p.A <= PL_SCALAR ? 1 : VEC, n = (p.A + vec - 1) / vec;     // vectors of a row
        // Lanes of a row, with up to 8 single elements or 4 vectors each (us; half as many / these / twice: 200000 x 32 fp32 41 / 34, 10 elements
        // 262144 x 18 42 / 40; 100000 x 300 fp32 176 / 129 / 133, 50000 x 100 bf16 27 / 26 / 33, 20000 x 1000 60 / 49 / 49).
        int G = 1;
        while (G < 64 && G * (vec == 1 ? 8 : 4) < n) G *= 2;
        const int64_t want = (p.B + NR_THREADS / G - 1) / (NR_THREADS / G);
        records = (int)(want < PL_RECORDS ? want : PL_RECORDS);
        const int H = (n + G - 1) / G;
        if (records == 1) { p.stats = out_stats; out_stats = nullptr; }
        if (vec == 1) {
            if (H <= 4) rows_go<T, KL, 1, 4>(p, G, records, s);
            else if (H <= 6) rows_go<T, KL, 1, 6>(p, G, records, s);
            else rows_go<T, KL, 1, 8>(p, G, records, s);
        } else if (H <= 2) rows_go<T, KL, VEC, 2>(p, G, records, s);
        else if (H <= 4) rows_go<T, KL, VEC, 4>(p, G, records, s);
        else rows_go<T, KL, VEC, PL_HELD>(p, G, records, s);
    } else {
        // Few long rows are split, into pieces of at least one vector a lane; a row that one workgroup gets through in about the time of
        // another launch is not (bf16, log-probabilities, split / not: 16 x 20000 11.5 / 7.9 us, x 100000 12.5 / 14.7, 256 x 100000 24.3 /
        // 21.6; the loss with the forward KL: 16 x 20000 20.6 / 17.8, x 100000 24.5 / 33.9, 256 x 100000 69.9 / 45.4).
        const int64_t pieces = (p.A + VEC * SP_THREADS - 1) / (VEC * SP_THREADS);
        int64_t splits = p.B < PL_SPLIT && (int64_t)p.A * (KL ? 2 : 1) > 32 * VEC * WR_THREADS ? 512 / p.B : 1;
        if (splits > pieces) splits = pieces;
        p.chunk = (int)((pieces + splits - 1) / splits * VEC * SP_THREADS);
        p.splits = (p.A + p.chunk - 1) / p.chunk;
        if (p.splits > 1) {
            records = (int)p.B;
            loss_parts_kernel<T, KL><<<dim3(p.splits, (unsigned)p.B), dim3(SP_THREADS), 0, s>>>(p);
            if (int rc = pl_launched(who)) return rc;
            if (p.g == p.z) {
                loss_border_kernel<T><<<dim3((unsigned)p.B), dim3(SP_THREADS), 0, s>>>(p);
                if (int rc = pl_launched(who)) return rc;
            } else {
                p.exact = nullptr;
            }
            if (KL == 0 && p.only_lp) loss_split_kernel<T, 0, false><<<dim3(1, (unsigned)p.B), dim3(SP_THREADS), 0, s>>>(p);
            else loss_split_kernel<T, KL, true><<<dim3(p.g ? p.splits : 1, (unsigned)p.B), dim3(SP_THREADS), 0, s>>>(p);
        } else {
            records = (int)(p.B < PL_RECORDS ? p.B : PL_RECORDS);
            const int per = p.A / (VEC * WR_THREADS);            // whole vectors a thread of 256: at least 2, and at least what the forms below hold in registers
            // With a gradient, the form that holds the most of the row (times in us, this line's form / the line's below, bf16; with a
            // reference the forward KL, with masks of each row's own four workgroups for longer: 6250 x 32000 478 / 393, 4000 x 50000 fp16 491 / 420).
            const bool own = p.mask && p.ldm;
            if constexpr (KL == 0) {
                // Log-probabilities: eight workgroups a compute unit, all 2048 of a pass at once (4096 x 32768 fp32 seven, whose second round is a few / eight
                // 94.5 / 85.6, 2000 x 150000 211 / 191, 10000 x 6000 fp16 49 / 38); bf16's take more registers than that leaves (8192 x 32000 110 / 133).
                constexpr int SIMD = __is_same(T, BF16) ? 4 : 8;
                if (p.only_lp && per >= 4) wide_go<T, KL, 4, 256, SIMD, 0, false>(p, records, s);
                else if (p.only_lp) wide_go<T, KL, 2, 256, SIMD, 0, false>(p, records, s);
                else if (p.g && per >= 96) wide_go<T, KL, 40, 512, 2, 16>(p, records, s);         // 887 x 225285 219 / 231, but 1148 x 174085 219 / 210
                else if (p.g && per >= 48) wide_go<T, KL, 40, 256, 2, 16>(p, records, s);    // 1953 x 102405 192 / 194, but 2325 x 86021 198 / 194
                else if (p.g && per >= 30) wide_go<T, KL, 20, 256, 2, 16>(p, records, s);    // 2500 x 80000 184 / 212, but 4000 x 50000 186 / 177
                else if (p.g && per >= 15) wide_go<T, KL, 15, 256, 4, 0>(p, records, s);     // 8192 x 32000 224 / 247, eight in registers and nine in LDS
                else if (p.g && per >= 8) wide_go<T, KL, 8, 256, 4, 0>(p, records, s);       // 8192 x 28000 181 / 215, but 8192 x 14000 105 / 104
                else if (per >= 4) wide_go<T, KL, 4, 256, 4, 0>(p, records, s);
                else wide_go<T, KL, 2, 256, 4, 0>(p, records, s);
            } else {
                if (p.g && per >= 44) wide_go<T, KL, 20, 512, 2, 8>(p, records, s);          // 1992 x 100357 forward 341 / 370, but 2325 x 86021 377 / 375
                else if (p.g && per >= (own ? 28 : 20)) wide_go<T, KL, 20, 256, 2, 8>(p, records, s);    // 4347 x 46000 277 / 316
                else if (p.g && per >= (own ? 28 : 15)) wide_go<T, KL, 12, 256, 2, 8>(p, records, s);    // 6259 x 31953 342 / 401, but 8000 x 25000 315 / 294
                else if (p.g && per >= 4) wide_go<T, KL, 4, 256, 4, 4>(p, records, s);       // 9523 x 21000 forward 294 / 338, 8192 x 8200 120 / 128
                else wide_go<T, KL, 2, 256, 4, 0>(p, records, s);
            }
        }
    }
    if (int rc = pl_launched(who)) return rc;
    if (!out_stats) return ACCERL_OK;
    loss_stats_kernel<<<dim3(1), dim3(records <= 256 ? 64 : 1024), 0, s>>>(p.rec, records, p.scale, out_stats);
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

constexpr int64_t PL_WORKSPACE = PL_RECORDS * (int64_t)sizeof(Record) + PL_PARTS * (int64_t)sizeof(Part) + PL_SPLIT * (int64_t)sizeof(double);
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
    p.exact = (double*)(p.part + PL_PARTS);
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
    const int es = dtype_bytes(a->dtype);
    if (!pl_aligned(a->old_logp, 4) || !pl_aligned(a->advantages, 4) || !pl_aligned(a->weights, 4) || !pl_aligned(a->ref_logp, 4) ||
        !pl_aligned(a->out_loss, 4) || !pl_aligned(a->out_logp, 4) || !pl_aligned(a->out_kl, 4) || !pl_aligned(a->out_entropy, 4) ||
        !pl_aligned(a->out_stats, 4) || !pl_aligned(a->grad_logits, es) || (ref && !pl_aligned(a->ref_logits, es)))
        return pl_fail(ACCERL_EINVAL, who, "misaligned argument");
    if (a->grad_logits) {
        const Table g = table(a->grad_logits, a->B, a->ld_grad, a->A, es);
        const bool in_place = a->grad_logits == a->logits && a->ld_grad == a->ld_logits;
        if (!in_place && share(g, table(a->logits, a->B, a->ld_logits, a->A, es)))
            return pl_fail(ACCERL_EINVAL, who, "the gradient overlaps the logits and is not the same table");
        if (ref && share(g, table(a->ref_logits, a->B, a->ld_ref, a->A, es))) return pl_fail(ACCERL_EINVAL, who, "the gradient overlaps the reference's logits");
    }
    LossParams p{};
    table_params(p, a->B, a->A, a->logits, a->ld_logits, a->mask, a->ld_mask, a->actions, a->workspace);
    p.zr = ref ? a->ref_logits : nullptr; p.ldr = a->ld_ref;
    p.g = a->grad_logits; p.ldg = a->ld_grad;
    p.old = a->old_logp; p.adv = a->advantages; p.w = a->weights; p.ref_lp = a->ref_logp;
    p.loss = a->out_loss; p.lp = a->out_logp; p.kl = a->out_kl; p.ent = a->out_entropy;
    p.kind = a->kl_kind;
    p.lo = 1.0 - a->clip_low; p.hi = 1.0 + a->clip_high;
    p.log_lo = (float)log(p.lo); p.log_hi = (float)log(p.hi);
    p.ck = (float)a->kl_coef; p.ch = (float)a->entropy_coef; p.scale = (float)a->scale;
    if (!a->out_stats) p.rec = nullptr;
    return loss_run(who, a->dtype, p, a->out_stats, (hipStream_t)stream);
}

}  // extern "C"
