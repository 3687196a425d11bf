// Linear attention with a decay for each head: unroll, gradients, single tokens.
//
// With E_i = d_i E_{i-1} + b_i c_i^T and out_i = a_i E_i ("a mixing of c by a and b"), everything here is the same operation:
//     out:     a = q,  b = k, c = v,  tokens forwards                 (E is the state S)
//     grad_q:  a = do, b = v, c = k,  forwards                        (E = S^T)
//     grad_v:  a = k,  b = q, c = do, from the last token to the first   (E is the gradient R of the state)
//     grad_k:  a = v,  b = do, c = q, backwards                       (E = R^T)
// A workgroup walks over a sequence in chunks of 64 tokens, for 64 columns of c.  Inside a chunk pairs of tokens meet directly,
//     out_t = sum_{s <= t} (a_t . b_s) g^{t-s} c_s  +  g^{t+1} a_t E_before,
// and the chunk's last state is g^64 E_before + sum_s g^{63-s} b_s c_s^T: four matrix products.
#include <algorithm>
#include <cstdio>

#include "wide_ops.h"

namespace accerl {
namespace {

constexpr int LC = 64;                    // tokens of a chunk: 16 for each wavefront
constexpr int LY = 64;                    // columns of c for a workgroup
constexpr float LOG2E = 1.44269504f;

typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));

struct LaSide { const void* p; int64_t sb, st, sh; int div; };                // [B, T, H / div, D]

struct LaRole {
    LaSide a, b, c;                       // a and b are X wide, c is Y wide
    void* out;                            // [B, T, H, Y] of the tokens' type, or fp32 (out_f32)
    int64_t ob, ot, oh;
    const float* enter;                   // the state before the first token of a segment, or NULL (zeros)
    float* last;                          // the state behind the last one, or NULL
    float* keep;                          // what is left of a segment's first state behind it, [segment][B H] (sums only)
    int64_t ex, ey, lx, ly;               // strides of x and y in both
    int64_t eseg, lseg;                   // from one segment's states to the next one's
    int X, Y, slices;
    int back;                             // from the last token to the first
    int out_f32;
    float pair, scale;                    // factors of b c^T and of out
};

struct LaParams {
    LaRole role[3];
    const float* log_decay;
    const uint8_t* reset;
    int64_t rb, rt;
    const int32_t* lengths;
    int64_t T, seg_len;                   // tokens of a segment, a multiple of LC
    int H, segs;
    uint32_t groups;                      // B H segs
};

// The element types of the matrix products: bf16 tokens as they are, others as fp32.
template <typename T> struct LaCompute { typedef float E; static constexpr bool HALF = false; };
template <> struct LaCompute<BF16> { typedef BF16 E; static constexpr bool HALF = true; };

__device__ __forceinline__ float pow2(float x) { return __builtin_amdgcn_exp2f(x); }
// g^n of lg = log2 g, which may be -inf
__device__ __forceinline__ float decay_pow(float lg, int n) { return n == 0 ? 1.0f : pow2(lg * (float)n); }

// 16 bytes of a row of which `left` elements are inside; the others are zeros
template <typename T> __device__ __forceinline__ u32x4 row_vec(const T* p, int left) {
    constexpr int N = 16 / sizeof(T);
    if (left >= N) {
        if constexpr (sizeof(T) == 4) return *(const u32x4_at4*)p;
        else return *(const u32x4_at2*)p;
    }
    u32x4 v = {0, 0, 0, 0};
    if (left > 0) {
        T e[N];
#pragma unroll
        for (int j = 0; j < N; ++j) e[j] = T{};
#pragma unroll
        for (int j = 0; j < N; ++j) if (j < left) e[j] = p[j];
        __builtin_memcpy(&v, e, 16);
    }
    return v;
}

// largest magnitude so far, as bits: halves of a word (bf16) or words
template <bool HALF> __device__ __forceinline__ void keep_top(uint32_t& top, uint32_t w) {
    if constexpr (HALF) {
        typedef unsigned short us2 __attribute__((ext_vector_type(2)));
        top = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(us2, top), __builtin_bit_cast(us2, w & 0x7fff7fffu)));
    } else {
        top = max(top, w & 0x7fffffffu);
    }
}
template <bool HALF> __device__ __forceinline__ bool not_finite(uint32_t top) {
    return HALF ? (top & 0xffffu) >= 0x7f80u || (top >> 16) >= 0x7f80u : top >= 0x7f800000u;
}

template <typename T, int DX>
struct LaTile {
    typedef typename LaCompute<T>::E E;
    static constexpr bool HALF = LaCompute<T>::HALF;
    // rows 16 bytes further on in the banks: a quarter wavefront's 16-byte reads of 16 rows meet no bank twice.  c is only read down its columns
    // (bf16: transposing reads of four rows, which 32 bytes keep apart)
    static constexpr int BP = DX + 16 / (int)sizeof(E);
    static constexpr int CP = HALF ? LY + 16 : LY + 4;
    static constexpr int VE = 16 / (int)sizeof(T);            // elements of a vector in memory
    static constexpr int BV = LC * DX / VE / 256, CV = LC * LY / VE / 256;
    static constexpr int FR = HALF ? 32 : 16;                 // depth of a fragment
    static constexpr int KX = DX / FR;
};

template <typename T, int DX, bool OUT>
__global__ __launch_bounds__(256, LaCompute<T>::HALF ? 2 : 1) void la_chunks_kernel(const LaParams p) {
    typedef LaTile<T, DX> L;
    typedef typename L::E E;
    constexpr bool HALF = L::HALF;
    constexpr int NA = DX / 64;                               // tiles of 16 rows of the state for a wavefront

    __shared__ __attribute__((aligned(16))) E sb[LC * L::BP];
    __shared__ __attribute__((aligned(16))) E sc[LC * L::CP];
    // the state as the fragments that the product with a reads: [column tile][depth][lane]
    __shared__ __attribute__((aligned(16))) E ss[OUT ? DX * LY : 16];
    __shared__ int odd[4];                                    // whether a wavefront has seen a NaN or an infinity in b or c
    __shared__ float red[4][LY];

    const int tid = threadIdx.x, w = tid >> 6, lane = tid & 63, g = lane >> 4, r = lane & 15;
    // workgroups go round the eight XCDs: the slices of a sequence, which read the same a and b, lie eight apart
    uint32_t id = blockIdx.x, which = 0, slice = 0;
    int slices = 0;
#pragma unroll
    for (int i = 0; i < 3; ++i) slices += p.role[i].slices;
    const uint32_t grp = id / (8 * slices) * 8 + id % 8;
    slice = id / 8 % slices;
    if (grp >= p.groups) return;
    while (slice >= (uint32_t)p.role[which].slices) slice -= p.role[which++].slices;
    const LaRole& q = p.role[which];
    const int X = q.X, Y = q.Y, y0 = slice * LY;
    const uint32_t seg = grp % p.segs, bh = grp / p.segs;
    const uint32_t b = bh / p.H, h = bh % p.H;
    const int back = q.back;

    int64_t n = p.T;
    if (p.lengths) n = min(max((int64_t)p.lengths[b], (int64_t)0), n);
    const int64_t i0 = seg * p.seg_len, i1 = min(n, i0 + p.seg_len);
    const float lg = p.log_decay[h] * LOG2E;
    const T* pa = (const T*)q.a.p + b * q.a.sb + (h / q.a.div) * q.a.sh;
    const T* pb = (const T*)q.b.p + b * q.b.sb + (h / q.b.div) * q.b.sh;
    const T* pc = (const T*)q.c.p + b * q.c.sb + (h / q.c.div) * q.c.sh + y0;
    const int yw = min(Y - y0, LY);                           // columns of the slice

    // the state: rows 16 (NA w + ta) + 4 g + i, columns 16 d + r
    v4f S[NA][4];
    {
        const float* e = q.enter ? q.enter + seg * q.eseg + (int64_t)bh * X * Y : nullptr;
#pragma unroll
        for (int ta = 0; ta < NA; ++ta)
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int x = 16 * (NA * w + ta) + 4 * g + i, y = y0 + 16 * d + r;
                    S[ta][d][i] = e && x < X && y < Y ? e[x * q.ex + y * q.ey] : 0.0f;
                }
    }
    // tables of a whole chunk: weights of pairs (tokens s = 16 st + 4 g + i, t = 16 w + r), of the state for token t, of token s for the state
    float dec[4][4], kw[4][4];
    const int t = 16 * w + r;
    float qw = decay_pow(lg, t + 1 - back);
#pragma unroll
    for (int st = 0; st < 4; ++st)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int s = 16 * st + 4 * g + i;
            dec[st][i] = s <= t ? decay_pow(lg, t - s) * q.pair : 0.0f;
            kw[st][i] = decay_pow(lg, LC - 1 - s + back) * q.pair;
        }
    float left = 1.0f;                                        // of the segment's first state

    u32x4 vb[L::BV], vc[L::CV];
    uint32_t cut = 0;
    auto token = [&](int64_t i) { return back ? n - 1 - i : i; };
    auto fetch = [&](int64_t base) {
#pragma unroll
        for (int k = 0; k < L::BV; ++k) {
            const int v = tid + 256 * k, row = v / (DX / L::VE), col = v % (DX / L::VE) * L::VE;
            const int64_t i = base + row;
            vb[k] = row_vec(pb + (i < i1 ? token(i) * q.b.st + col : 0), i < i1 ? X - col : 0);
        }
#pragma unroll
        for (int k = 0; k < L::CV; ++k) {
            const int v = tid + 256 * k, row = v / (LY / L::VE), col = v % (LY / L::VE) * L::VE;
            const int64_t i = base + row;
            vc[k] = row_vec(pc + (i < i1 ? token(i) * q.c.st + col : 0), i < i1 ? yw - col : 0);
        }
        // does token i = base + lane start from nothing?  (backwards: does the token before it in this order, the one behind it)
        cut = 0;
        if (p.reset) {
            const int64_t i = base + lane, at = back ? n - i : i;
            if (i < i1 && !(back && i == 0)) cut = p.reset[b * p.rb + at * p.rt];
        }
    };
    auto stage = [&]() {
        uint32_t top = 0;
        auto put = [&](E* to, u32x4 v) {
            if constexpr (__is_same(T, F16)) {
                float f[8];
#pragma unroll
                for (int j = 0; j < 4; ++j) el_pair<F16>(v[j], f[2 * j], f[2 * j + 1]);
#pragma unroll
                for (int j = 0; j < 8; ++j) keep_top<false>(top, __float_as_uint(f[j]));
                *(v4f*)to = v4f{f[0], f[1], f[2], f[3]};
                *(v4f*)(to + 4) = v4f{f[4], f[5], f[6], f[7]};
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) keep_top<HALF>(top, v[j]);
                *(u32x4*)to = v;
            }
        };
#pragma unroll
        for (int k = 0; k < L::BV; ++k) {
            const int v = tid + 256 * k;
            put(sb + v / (DX / L::VE) * L::BP + v % (DX / L::VE) * L::VE, vb[k]);
        }
#pragma unroll
        for (int k = 0; k < L::CV; ++k) {
            const int v = tid + 256 * k;
            put(sc + v / (LY / L::VE) * L::CP + v % (LY / L::VE) * L::VE, vc[k]);
        }
        const bool any = __ballot(not_finite<HALF>(top)) != 0;
        if (lane == 0) odd[w] = any;
    };
    auto publish = [&]() {
        if constexpr (OUT)
#pragma unroll
            for (int ta = 0; ta < NA; ++ta) {
                const int at = NA * w + ta;
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    if constexpr (HALF) {                     // depth 32: rows 4 quad .. of the 32 belong to lane group quad / 2
                        const int quad = 4 * (at & 1) + g;
                        u32x2 two = {f32_pair<BF16>(S[ta][d][0], S[ta][d][1]), f32_pair<BF16>(S[ta][d][2], S[ta][d][3])};
                        *(u32x2*)(ss + ((d * L::KX + (at >> 1)) * 64 + 16 * (quad >> 1) + r) * 8 + 4 * (quad & 1)) = two;
                    } else {
                        *(v4f*)(ss + ((d * L::KX + at) * 64 + lane) * 4) = S[ta][d];
                    }
                }
            }
    };
    auto out_at = [&](int64_t i) { return b * q.ob + (int64_t)h * q.oh + token(i) * q.ot + y0; };

    if (i0 < i1) { fetch(i0); stage(); publish(); }
    for (int64_t base = i0; base < i1; base += LC) {
        const int m = (int)min((int64_t)LC, i1 - base);
        const uint64_t cuts = __ballot(cut != 0);
        __syncthreads();
        const bool more = base + LC < i1;
        if (more) fetch(base + LC);
        const bool plain = !(odd[0] | odd[1] | odd[2] | odd[3]);
        if (m < LC) {
#pragma unroll
            for (int st = 0; st < 4; ++st)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int s = 16 * st + 4 * g + i;
                    kw[st][i] = s < m ? decay_pow(lg, m - 1 - s + back) * q.pair : 0.0f;
                }
        }
        const int last_cut = cuts ? 63 - __builtin_clzll(cuts) : -1;
        const uint64_t before = cuts & ((2ull << t) - 1);
        const int first = before ? 63 - __builtin_clzll(before) : -1;        // the token that t's episode begins with, if it begins in this chunk

        if (plain) {
            v4f O[4];
            E pt[4][4];                                       // weights of pairs as the product with c reads them
            if constexpr (OUT) {
                // this wavefront's 16 tokens of a, straight from memory
                const bool have = t < m;
                const T* ra = pa + (have ? token(base + t) * q.a.st : 0);
#pragma unroll
                for (int d = 0; d < 4; ++d) O[d] = v4f{0, 0, 0, 0};
                v4f P[4];
#pragma unroll
                for (int st = 0; st < 4; ++st) P[st] = v4f{0, 0, 0, 0};
                if constexpr (HALF) {
                    v8bf fa[L::KX];
#pragma unroll
                    for (int k = 0; k < L::KX; ++k) fa[k] = __builtin_bit_cast(v8bf, row_vec(ra + (have ? 32 * k + 8 * g : 0), have ? X - 32 * k - 8 * g : 0));
#pragma unroll
                    for (int st = 0; st < 4; ++st)
                        if (st <= w)
#pragma unroll
                            for (int k = 0; k < L::KX; ++k)
                                P[st] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*(const v8bf*)(sb + (16 * st + r) * L::BP + 32 * k + 8 * g), fa[k], P[st], 0, 0, 0);
#pragma unroll
                    for (int k = 0; k < L::KX; ++k)
#pragma unroll
                        for (int d = 0; d < 4; ++d)
                            O[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*(const v8bf*)(ss + ((d * L::KX + k) * 64 + lane) * 8), fa[k], O[d], 0, 0, 0);
                } else {
                    for (int k = 0; k < L::KX; ++k) {
                        v4f fa = {0, 0, 0, 0};
                        const int in = have ? X - 16 * k - 4 * g : 0;
                        const T* rk = ra + (in > 0 ? 16 * k + 4 * g : 0);
                        if constexpr (sizeof(T) == 4) fa = __builtin_bit_cast(v4f, row_vec(rk, in));
                        else
#pragma unroll
                            for (int j = 0; j < 4; ++j) if (j < in) fa[j] = el_f32(rk[j]);
#pragma unroll
                        for (int st = 0; st < 4; ++st)
                            if (st <= w) {
                                const v4f fb = *(const v4f*)(sb + (16 * st + r) * L::BP + 16 * k + 4 * g);
#pragma unroll
                                for (int j = 0; j < 4; ++j) P[st] = __builtin_amdgcn_mfma_f32_16x16x4f32(fb[j], fa[j], P[st], 0, 0, 0);
                            }
#pragma unroll
                        for (int d = 0; d < 4; ++d) {
                            const v4f fs = *(const v4f*)(ss + ((d * L::KX + k) * 64 + lane) * 4);
#pragma unroll
                            for (int j = 0; j < 4; ++j) O[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(fs[j], fa[j], O[d], 0, 0, 0);
                        }
                    }
                }
                // (selected, not multiplied by 0: the state of the episode before may hold anything)
                const float f = qw;
#pragma unroll
                for (int d = 0; d < 4; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i) O[d][i] = first >= 0 ? 0.0f : O[d][i] * f;
#pragma unroll
                for (int st = 0; st < 4; ++st)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int s = 16 * st + 4 * g + i;
                        pt[st][i] = f32_el<E>(s <= t && s >= first ? P[st][i] * dec[st][i] : 0.0f);
                    }
            }
            // what enters the next chunk
            const float sd = decay_pow(lg, m);
#pragma unroll
            for (int ta = 0; ta < NA; ++ta)
#pragma unroll
                for (int d = 0; d < 4; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i) S[ta][d][i] = cuts ? 0.0f : S[ta][d][i] * sd;
            if constexpr (HALF) {
#pragma unroll
                for (int ks = 0; ks < 2; ++ks) {
                    // four rows of four columns each are turned by a read: the columns of 16 lanes, down four tokens
                    typedef __attribute__((address_space(3))) v4s lds4;
                    auto down = [&](const E* tile, int pitch, int col) {
                        const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(tile + (32 * ks + 4 * g + (r >> 2)) * pitch + col + 4 * (r & 3)));
                        const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(tile + (32 * ks + 16 + 4 * g + (r >> 2)) * pitch + col + 4 * (r & 3)));
                        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                    };
                    v8bf fc[4];
#pragma unroll
                    for (int d = 0; d < 4; ++d) fc[d] = __builtin_bit_cast(v8bf, down(sc, L::CP, 16 * d));
                    if constexpr (OUT) if (2 * ks <= w) {
                        v8s pp;
#pragma unroll
                        for (int j = 0; j < 8; ++j) pp[j] = (short)pt[2 * ks + j / 4][j % 4].u;
#pragma unroll
                        for (int d = 0; d < 4; ++d) O[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fc[d], __builtin_bit_cast(v8bf, pp), O[d], 0, 0, 0);
                    }
#pragma unroll
                    for (int ta = 0; ta < NA; ++ta) {
                        // b weighted in fp32 and split in two bf16 parts: the state keeps 2^-17 of every term
                        const v8s fb = down(sb, L::BP, 16 * (NA * w + ta));
                        v8s hi, lo;
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const int s = 32 * ks + (j < 4 ? 0 : 16) + 4 * g + j % 4;
                            const float x = el_f32(BF16{(uint16_t)fb[j]}) * kw[2 * ks + j / 4][j % 4];
                            const float xw = s < last_cut ? 0.0f : x;
                            const BF16 xh = f32_el<BF16>(xw);
                            hi[j] = (short)xh.u;
                            lo[j] = (short)f32_el<BF16>(xw - el_f32(xh)).u;
                        }
#pragma unroll
                        for (int d = 0; d < 4; ++d) {
                            S[ta][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, lo), fc[d], S[ta][d], 0, 0, 0);
                            S[ta][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, hi), fc[d], S[ta][d], 0, 0, 0);
                        }
                    }
                }
            } else {
#pragma unroll
                for (int st = 0; st < 4; ++st) {
                    v4f fc[4];
#pragma unroll
                    for (int d = 0; d < 4; ++d)
#pragma unroll
                        for (int i = 0; i < 4; ++i) fc[d][i] = sc[(16 * st + 4 * g + i) * L::CP + 16 * d + r];
                    if constexpr (OUT) if (st <= w) {
#pragma unroll
                        for (int d = 0; d < 4; ++d)
#pragma unroll
                            for (int i = 0; i < 4; ++i) O[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(fc[d][i], pt[st][i], O[d], 0, 0, 0);
                    }
#pragma unroll
                    for (int ta = 0; ta < NA; ++ta)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int s = 16 * st + 4 * g + i;
                            const float x = sb[s * L::BP + 16 * (NA * w + ta) + r] * kw[st][i];
                            const float xw = s < last_cut ? 0.0f : x;
#pragma unroll
                            for (int d = 0; d < 4; ++d) S[ta][d] = __builtin_amdgcn_mfma_f32_16x16x4f32(xw, fc[d][i], S[ta][d], 0, 0, 0);
                        }
                }
            }
            if constexpr (OUT) {
                if (t < m) {
                    const int64_t o = out_at(base + t);
#pragma unroll
                    for (int d = 0; d < 4; ++d) {
                        const int y = 16 * d + 4 * g;
                        v4f v = O[d];
#pragma unroll
                        for (int i = 0; i < 4; ++i) v[i] *= q.scale;
                        if (q.out_f32) {
                            float* to = (float*)q.out + o + y;
                            if (y + 4 <= yw) *(u32x4_at4*)to = __builtin_bit_cast(u32x4, v);
                            else
#pragma unroll
                                for (int i = 0; i < 4; ++i) if (y + i < yw) to[i] = v[i];
                        } else {
                            T* to = (T*)q.out + o + y;
                            if (y + 4 <= yw) {
                                if constexpr (sizeof(T) == 4) *(u32x4_at4*)to = __builtin_bit_cast(u32x4, v);
                                else *(u32x2_at2*)to = u32x2{f32_pair<T>(v[0], v[1]), f32_pair<T>(v[2], v[3])};
                            } else
#pragma unroll
                                for (int i = 0; i < 4; ++i) if (y + i < yw) to[i] = f32_el<T>(v[i]);
                        }
                    }
                }
            }
        } else {
            // A NaN or an infinity in the chunk: in the products above a weight of 0 would carry it to tokens before it and to other episodes.  Token by token,
            // as the formula says.
            const float ge = pow2(lg);
            for (int s = 0; s < m; ++s) {
                const bool anew = cuts >> s & 1;
                float part[4] = {0, 0, 0, 0};
#pragma unroll
                for (int ta = 0; ta < NA; ++ta)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int x = 16 * (NA * w + ta) + 4 * g + i;
                        const float eb = el_f32(sb[s * L::BP + x]) * q.pair;
                        float ea = 0.0f;
                        if constexpr (OUT) if (x < X) ea = el_f32(pa[token(base + s) * q.a.st + x]);
#pragma unroll
                        for (int d = 0; d < 4; ++d) {
                            float e = anew ? 0.0f : back ? S[ta][d][i] : S[ta][d][i] * ge;
                            e += eb * el_f32(sc[s * L::CP + 16 * d + r]);
                            if (x < X) part[d] += ea * e;
                            S[ta][d][i] = back ? e * ge : e;
                        }
                    }
                if constexpr (OUT) {
#pragma unroll
                    for (int d = 0; d < 4; ++d) {
                        part[d] += __shfl_xor(part[d], 16);
                        part[d] += __shfl_xor(part[d], 32);
                        if (g == 0) red[w][16 * d + r] = part[d];
                    }
                    __syncthreads();
                    if (tid < yw) {
                        const float v = (red[0][tid] + red[1][tid] + red[2][tid] + red[3][tid]) * q.scale;
                        const int64_t o = out_at(base + s) + tid;
                        if (q.out_f32) ((float*)q.out)[o] = v;
                        else ((T*)q.out)[o] = f32_el<T>(v);
                    }
                    __syncthreads();
                }
            }
        }
        left = cuts ? 0.0f : left * decay_pow(lg, m);
        __syncthreads();
        if (more) { stage(); publish(); }
    }

    if (q.last) {
        // backwards the state that enters the unroll has no gradient if its first token resets
        const bool gone = back && seg == p.segs - 1 && n > 0 && p.reset && p.reset[b * p.rb] != 0;
        if (gone) left = 0.0f;
        float* e = q.last + seg * q.lseg + (int64_t)bh * X * Y;
#pragma unroll
        for (int ta = 0; ta < NA; ++ta)
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int x = 16 * (NA * w + ta) + 4 * g + i, y = y0 + 16 * d + r;
                    if (x < X && y < Y) e[x * q.lx + y * q.ly] = gone ? 0.0f : S[ta][d][i];
                }
        if (q.keep && slice == 0 && tid == 0) q.keep[(int64_t)seg * (p.groups / p.segs) + bh] = left;
    }
    if constexpr (OUT) {
        // tokens behind the sequence's end
        for (int64_t i = max(i0, n) + w; i < min(p.T, i0 + p.seg_len); i += 4) {
            const int64_t o = b * q.ob + (int64_t)h * q.oh + i * q.ot + y0;
            if (lane < yw) {
                if (q.out_f32) ((float*)q.out)[o + lane] = 0.0f;
                else ((T*)q.out)[o + lane] = T{};
            }
        }
    }
}

// The states that enter the segments, from what each segment adds: states [segment][B H][X Y] in place, the last one to `last`.
struct LaJoin { float* states; const float* keep; const float* enter; float* last; };
struct LaJoinParams { LaJoin at[2]; int64_t n, per; int segs; };               // n = B H X Y, per = X Y
__global__ __launch_bounds__(256) void la_join_kernel(const LaJoinParams p) {
    const LaJoin& j = p.at[blockIdx.y];
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= p.n) return;
    const int64_t bh = i / p.per, all = p.n / p.per;
    float e = j.enter ? j.enter[i] : 0.0f;
    for (int s = 0; s < p.segs; ++s) {
        const float add = j.states[s * p.n + i], f = j.keep[s * all + bh];
        j.states[s * p.n + i] = e;
        e = (f == 0.0f ? 0.0f : f * e) + add;
    }
    if (j.last) j.last[i] = e;
}

// The gradients of shared keys and values: the heads' parts [B, T, H, D] in fp32, summed in the heads' order and rounded once.
struct LaFold { const float* part; void* out; int64_t sb, st, sh; int D; };
struct LaFoldParams { LaFold at[2]; int64_t tokens, T; int H, Hk; };
template <typename T>
__global__ __launch_bounds__(256) void la_fold_kernel(const LaFoldParams p) {
    const LaFold& f = p.at[blockIdx.y];
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= p.tokens * p.Hk * f.D) return;
    const int x = (int)(i % f.D), share = p.H / p.Hk;
    const int64_t row = i / f.D, token = row / p.Hk, hk = row % p.Hk, b = token / p.T;
    const float* from = f.part + (token * p.H + hk * share) * f.D + x;
    float s = 0.0f;
    for (int k = 0; k < share; ++k) s += from[(int64_t)k * f.D];
    ((T*)f.out)[b * f.sb + (token - b * p.T) * f.st + hk * f.sh + x] = f32_el<T>(s);
}

// ---------------------------------------------------------------- single tokens
struct LaStep {
    LaSide q, k, v;
    void* out;
    int64_t ob, oh;
    const float* log_decay;
    const uint8_t* reset;
    int64_t rb;
    const float* state;
    float* out_state;
    float scale;
    int H, X, Y, slices;
};

// A workgroup has 64 columns of a state: 16 lanes of four columns, 16 rows at a time, all rows asked for before the first is used.  Bound by memory: the state
// is read and written once.
template <typename T, int ROWS>
__global__ __launch_bounds__(256) void la_step_kernel(const LaStep p) {
    __shared__ v4f red[4][16];
    const int tid = threadIdx.x, w = tid >> 6, lane = tid & 63, r = lane & 15, x0 = tid >> 4;
    const uint32_t slice = blockIdx.x % p.slices, bh = blockIdx.x / p.slices, b = bh / p.H, h = bh % p.H;
    const int y = slice * 64 + 4 * r, in = min(max(p.Y - y, 0), 4);
    const bool anew = p.reset && p.reset[b * p.rb] != 0;
    const T* pq = (const T*)p.q.p + b * p.q.sb + h * p.q.sh;
    const T* pk = (const T*)p.k.p + b * p.k.sb + (h / p.k.div) * p.k.sh;
    const T* pv = (const T*)p.v.p + b * p.v.sb + (h / p.v.div) * p.v.sh + y;
    const float* s = p.state + (int64_t)bh * p.X * p.Y;
    float* so = p.out_state + (int64_t)bh * p.X * p.Y;
    v4f S[ROWS];
    float k[ROWS], q[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int x = x0 + 16 * i;
        S[i] = v4f{0, 0, 0, 0};
        k[i] = q[i] = 0.0f;
        if (x < p.X) {
            if (!anew) S[i] = __builtin_bit_cast(v4f, row_vec(s + (int64_t)x * p.Y + (in ? y : 0), in));
            k[i] = el_f32(pk[x]);
            q[i] = el_f32(pq[x]);
        }
    }
    v4f v = {0, 0, 0, 0}, o = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < 4; ++j) if (j < in) v[j] = el_f32(pv[j]);
    const float ge = pow2(p.log_decay[h] * LOG2E);
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int x = x0 + 16 * i;
        if (x < p.X) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                S[i][j] = (anew ? 0.0f : ge * S[i][j]) + k[i] * v[j];
                o[j] += q[i] * S[i][j];
            }
            float* to = so + (int64_t)x * p.Y + y;
            if (in == 4) *(u32x4_at4*)to = __builtin_bit_cast(u32x4, S[i]);
            else
#pragma unroll
                for (int j = 0; j < 4; ++j) if (j < in) to[j] = S[i][j];
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        o[j] += __shfl_xor(o[j], 16);
        o[j] += __shfl_xor(o[j], 32);
    }
    if (lane < 16) red[w][r] = o;
    __syncthreads();
    if (tid < 16) {
        T* to = (T*)p.out + b * p.ob + h * p.oh + y;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < in) to[j] = f32_el<T>((red[0][r][j] + red[1][r][j] + red[2][r][j] + red[3][r][j]) * p.scale);
    }
}

// ---------------------------------------------------------------- host
int la_fail(int code, const char* who, const char* what) {
    char msg[160];
    snprintf(msg, sizeof msg, "%s: %s", who, what);
    return set_error(code, msg);
}
int la_launched(const char* who) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? ACCERL_OK : la_fail(ACCERL_EHIP, who, hipGetErrorString(e));
}
bool la_aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

constexpr int LA_MAX_D = 256;

struct LaPlan { int segs; int64_t seg_len; };
// Segments of a sequence, worked on side by side: what each adds to the state is summed first (keys and values are read twice), where sequences, heads and
// columns alone leave compute units without work.
LaPlan la_plan(int64_t B, int64_t T, int H, int slices) {
    const int64_t blocks = B * H * slices;
    int64_t segs = 1;
    if (blocks > 0 && blocks < 512 && T > 4 * LC) segs = std::max<int64_t>(1, std::min<int64_t>((1024 + blocks - 1) / blocks, T / (2 * LC)));
    const int64_t chunks = (T + LC - 1) / LC;
    const int64_t per = std::max<int64_t>(1, (chunks + segs - 1) / segs);
    return {(int)std::max<int64_t>(1, (chunks + per - 1) / per), per * LC};
}
int la_slices(int y) { return (y + LY - 1) / LY; }
int64_t la_up(int64_t n) { return (n + 15) / 16 * 16; }

// floats of the workspace: the segments' states and what each keeps, for the state and (gradients) its gradient; the parts of shared gradients
struct LaWork { LaPlan plan; int64_t states, keep, parts_k, parts_v, total; };
LaWork la_work(int64_t B, int64_t T, int H, int Hk, int Dk, int Dv, bool grad) {
    LaWork k{};
    k.plan = la_plan(B, T, H, grad ? 2 * la_slices(Dk) + la_slices(Dv) : la_slices(Dv));
    if (k.plan.segs > 1) {
        k.states = la_up(B * H * (int64_t)Dk * Dv * k.plan.segs);
        k.keep = la_up(B * H * k.plan.segs);
    }
    if (grad && H != Hk) { k.parts_k = la_up(B * T * H * Dk); k.parts_v = la_up(B * T * H * Dv); }
    k.total = (grad ? 2 : 1) * (k.states + k.keep) + k.parts_k + k.parts_v;
    return k;
}

int la_check_sizes(const char* who, int64_t B, int64_t T, int32_t H, int32_t Hk, int32_t Dk, int32_t Dv) {
    if (B < 0 || T < 0 || H < 1 || Hk < 1 || Dk < 1 || Dv < 1) return la_fail(ACCERL_EINVAL, who, "need B, T >= 0 and H, Hk, Dk, Dv >= 1");
    if (H % Hk) return la_fail(ACCERL_EINVAL, who, "the heads of queries must be a multiple of those of keys and values");
    if (Dk > LA_MAX_D || Dv > LA_MAX_D) return la_fail(ACCERL_EUNSUPPORTED, who, "heads of more than 256 elements");
    if (H > (1 << 16) || B > ((int64_t)1 << 20) || B * H > ((int64_t)1 << 22) || T > ((int64_t)1 << 31) || B * T > ((int64_t)1 << 40)) return la_fail(ACCERL_EUNSUPPORTED, who, "more than 2^22 heads in all or 2^31 tokens");
    return ACCERL_OK;
}

template <typename T, bool OUT>
int la_launch(const char* who, const LaParams& p, int X, hipStream_t s) {
    int slices = 0;
    for (const LaRole& r : p.role) slices += r.slices;
    const int64_t blocks = ((int64_t)p.groups + 7) / 8 * 8 * slices;
    if (blocks * 256 > MAX_LAUNCH_ITEMS) return la_fail(ACCERL_EUNSUPPORTED, who, "more heads, segments and columns than one launch takes");
    const dim3 grid((uint32_t)blocks), block(256);
    if (X <= 64) la_chunks_kernel<T, 64, OUT><<<grid, block, 0, s>>>(p);
    else if (X <= 128) la_chunks_kernel<T, 128, OUT><<<grid, block, 0, s>>>(p);
    else la_chunks_kernel<T, 256, OUT><<<grid, block, 0, s>>>(p);
    return la_launched(who);
}
int la_pad(int x) { return x <= 64 ? 64 : x <= 128 ? 128 : 256; }

// launches of the roles, those of one width together
template <typename T, bool OUT>
int la_run(const char* who, const LaParams& common, const LaRole* roles, int count, hipStream_t s) {
    for (int x : {64, 128, 256}) {
        LaParams p = common;
        int n = 0;
        for (int i = 0; i < count; ++i) if (la_pad(roles[i].X) == x) p.role[n++] = roles[i];
        if (n) if (int rc = la_launch<T, OUT>(who, p, x, s)) return rc;
    }
    return ACCERL_OK;
}

LaSide la_side(const void* p, const accerl_token_stride& s, int div) { return {p, s.batch, s.token, s.head, div}; }

template <typename T>
int la_forward(const char* who, const accerl_linear_attention_args& a, LaParams p, const LaWork& k, float* ws, hipStream_t s) {
    const int share = a.H / a.Hk;
    const int64_t per = (int64_t)a.Dk * a.Dv, n = a.B * a.H * per;
    LaRole r{};
    r.a = la_side(a.q, a.q_stride, 1); r.b = la_side(a.k, a.k_stride, share); r.c = la_side(a.v, a.v_stride, share);
    r.X = a.Dk; r.Y = a.Dv; r.slices = la_slices(a.Dv);
    r.ex = r.lx = a.Dv; r.ey = r.ly = 1;
    r.pair = 1.0f; r.scale = (float)a.scale;
    if (p.segs > 1) {
        LaRole sum = r;
        sum.last = ws; sum.lseg = n; sum.keep = ws + k.states;
        if (int rc = la_run<T, false>(who, p, &sum, 1, s)) return rc;
        LaJoinParams j{};
        j.at[0] = {ws, ws + k.states, a.state, a.out_state};
        j.n = n; j.per = per; j.segs = p.segs;
        la_join_kernel<<<dim3((uint32_t)((n + 255) / 256)), dim3(256), 0, s>>>(j);
        if (int rc = la_launched(who)) return rc;
        r.enter = ws; r.eseg = n;
    } else {
        r.enter = a.state;
        r.last = a.out_state;
    }
    r.out = a.out; r.ob = a.out_stride.batch; r.ot = a.out_stride.token; r.oh = a.out_stride.head;
    return la_run<T, true>(who, p, &r, 1, s);
}

template <typename T>
int la_backward(const char* who, const accerl_linear_attention_args& a, LaParams p, const LaWork& k, float* ws, hipStream_t s) {
    const int share = a.H / a.Hk;
    const int64_t per = (int64_t)a.Dk * a.Dv, n = a.B * a.H * per;
    const LaSide q = la_side(a.q, a.q_stride, 1), key = la_side(a.k, a.k_stride, share), v = la_side(a.v, a.v_stride, share), go = la_side(a.grad_out, a.grad_out_stride, 1);
    const float scale = (float)a.scale;
    LaRole rq{}, rk{}, rv{};
    rq.a = go; rq.b = v; rq.c = key; rq.X = a.Dv; rq.Y = a.Dk; rq.ex = 1; rq.ey = a.Dv; rq.pair = 1.0f; rq.scale = scale;
    rk.a = v; rk.b = go; rk.c = q; rk.X = a.Dv; rk.Y = a.Dk; rk.ex = 1; rk.ey = a.Dv; rk.back = 1; rk.pair = scale; rk.scale = 1.0f;
    rv.a = key; rv.b = q; rv.c = go; rv.X = a.Dk; rv.Y = a.Dv; rv.ex = a.Dv; rv.ey = 1; rv.back = 1; rv.pair = scale; rv.scale = 1.0f;
    for (LaRole* r : {&rq, &rk, &rv}) { r->lx = r->ex; r->ly = r->ey; r->slices = la_slices(r->Y); }
    float *S = ws, *R = S + k.states, *keep = R + k.states, *keep_back = keep + k.keep, *parts_k = keep_back + k.keep, *parts_v = parts_k + k.parts_k;
    if (p.segs > 1) {
        LaRole sum[2] = {rq, rv};
        sum[0].b = key; sum[0].c = v;                          // the state itself, summed as the unroll sums it
        sum[0].X = a.Dk; sum[0].Y = a.Dv; sum[0].slices = la_slices(a.Dv);
        sum[0].lx = a.Dv; sum[0].ly = 1;
        sum[0].last = S; sum[0].keep = keep;
        sum[1].last = R; sum[1].keep = keep_back;
        for (LaRole& r : sum) r.lseg = n;
        if (int rc = la_run<T, false>(who, p, sum, 2, s)) return rc;
        LaJoinParams j{};
        j.at[0] = {S, keep, a.state, nullptr};
        j.at[1] = {R, keep_back, a.grad_out_state, a.grad_state};
        j.n = n; j.per = per; j.segs = p.segs;
        la_join_kernel<<<dim3((uint32_t)((n + 255) / 256), 2), dim3(256), 0, s>>>(j);
        if (int rc = la_launched(who)) return rc;
        rq.enter = S; rk.enter = rv.enter = R;
        rq.eseg = rk.eseg = rv.eseg = n;
    } else {
        rq.enter = a.state; rk.enter = rv.enter = a.grad_out_state;
        rv.last = a.grad_state;
    }
    auto to = [](LaRole& r, void* out, const accerl_token_stride& st) { r.out = out; r.ob = st.batch; r.ot = st.token; r.oh = st.head; };
    to(rq, a.grad_q, a.grad_q_stride);
    if (share == 1) {
        to(rk, a.grad_k, a.grad_k_stride);
        to(rv, a.grad_v, a.grad_v_stride);
    } else {
        to(rk, parts_k, {a.T * a.H * a.Dk, (int64_t)a.H * a.Dk, a.Dk});
        to(rv, parts_v, {a.T * a.H * a.Dv, (int64_t)a.H * a.Dv, a.Dv});
        rk.out_f32 = rv.out_f32 = 1;
    }
    LaRole roles[3] = {rq, rk, rv};
    if (int rc = la_run<T, true>(who, p, roles, 3, s)) return rc;
    if (share > 1) {
        LaFoldParams f{};
        f.at[0] = {parts_k, a.grad_k, a.grad_k_stride.batch, a.grad_k_stride.token, a.grad_k_stride.head, a.Dk};
        f.at[1] = {parts_v, a.grad_v, a.grad_v_stride.batch, a.grad_v_stride.token, a.grad_v_stride.head, a.Dv};
        f.tokens = a.B * a.T; f.T = a.T; f.H = a.H; f.Hk = a.Hk;
        const int64_t items = f.tokens * a.Hk * std::max(a.Dk, a.Dv);
        if (items > MAX_LAUNCH_ITEMS) return la_fail(ACCERL_EUNSUPPORTED, who, "more gradients of shared heads than one launch takes");
        la_fold_kernel<T><<<dim3((uint32_t)((items + 255) / 256), 2), dim3(256), 0, s>>>(f);
        if (int rc = la_launched(who)) return rc;
    }
    return ACCERL_OK;
}

// what all calls check, of one token (step) or many; `done` is set where nothing is to be done
int la_check(const char* who, const accerl_linear_attention_args* a, bool step, bool* done) {
    *done = false;
    if (!a) return la_fail(ACCERL_EINVAL, who, "NULL argument");
    if (!dtype_known(a->dtype)) return la_fail(ACCERL_EINVAL, who, "unknown type of tokens");
    if (int rc = la_check_sizes(who, a->B, step ? 1 : a->T, a->H, a->Hk, a->Dk, a->Dv)) return rc;
    if (!(a->scale > -1e30 && a->scale < 1e30)) return la_fail(ACCERL_EINVAL, who, "the scale must be finite");
    if (a->B == 0) { *done = true; return ACCERL_OK; }
    if (!a->log_decay || !la_aligned(a->log_decay, 4)) return la_fail(ACCERL_EINVAL, who, "log_decay is NULL or misaligned");
    if (!step && a->T == 0) return ACCERL_OK;
    const int e = dtype_bytes(a->dtype);
    for (const void* p : {a->q, a->k, a->v}) if (!p || !la_aligned(p, e)) return la_fail(ACCERL_EINVAL, who, "q, k or v is NULL or misaligned");
    if (!la_aligned(a->lengths, 4)) return la_fail(ACCERL_EINVAL, who, "misaligned lengths");
    return ACCERL_OK;
}
bool la_state_ok(const void* p) { return la_aligned(p, 16); }

// an output's own places: no two of them the same, as far as they are laid out in one of the orders of batch, token and head
bool la_spread(const accerl_token_stride& s, int64_t B, int64_t T, int H, int D) {
    if (s.batch < 0 || s.token < 0 || s.head < 0) return false;
    int64_t size[3] = {B, T, H}, step[3] = {s.batch, s.token, s.head};
    int order[3] = {0, 1, 2};
    std::sort(order, order + 3, [&](int x, int y) { return step[x] < step[y]; });
    __int128 reach = D;
    for (int i : order) {
        if (size[i] <= 1) continue;
        if (step[i] < reach) return false;
        reach += (__int128)step[i] * (size[i] - 1);
    }
    return true;
}

// A tensor of tokens as a table of rows, if its dimensions fold into one (contiguous heads or tokens, one stride over the rest).
bool la_table(const void* at, const accerl_token_stride& st, int64_t B, int64_t T, int64_t H, int D, int e, Table& t) {
    struct Dim { int64_t n, step; } d[3] = {{B, st.batch}, {T, st.token}, {H, st.head}};
    std::sort(d, d + 3, [](const Dim& x, const Dim& y) { return x.step < y.step; });
    int64_t run = D, rows = 1, apart = 0;
    for (const Dim& x : d) {
        if (x.n <= 1) continue;
        if (x.step < 0) return false;
        if (rows == 1 && x.step == run) run *= x.n;
        else if (rows == 1) { if (x.step < run) return false; rows = x.n; apart = x.step; }
        else if (x.step == apart * rows) rows *= x.n;
        else return false;
    }
    t = {at, rows, (rows == 1 ? run : apart) * e, run * e};
    return true;
}
// Whether an output shares elements with another tensor: looked for where both fold into tables (or at all where they lie apart), else the caller's to avoid.
struct LaTensor { const void* p; accerl_token_stride st; int H, D; };
bool la_overlap(const LaTensor& o, const LaTensor& t, int64_t B, int64_t T, int e) {
    Table a, b;
    return o.p && t.p && la_table(o.p, o.st, B, T, o.H, o.D, e, a) && la_table(t.p, t.st, B, T, t.H, t.D, e, b) && share(a, b);
}
bool la_states_overlap(const void* a, const void* b, const accerl_linear_attention_args* s) {
    const int64_t n = 4 * s->B * s->H * s->Dk * s->Dv;
    return a && b && share(table(a, n), table(b, n));
}

int la_workspace(const char* who, const accerl_linear_attention_args* a, const LaWork& k) {
    if (k.total == 0) return ACCERL_OK;
    if (!a->workspace || !la_aligned(a->workspace, 16)) return la_fail(ACCERL_EINVAL, who, "workspace is NULL or misaligned");
    if (a->workspace_bytes < 4 * k.total) return la_fail(ACCERL_EINVAL, who, "workspace smaller than accerl_linear_attention_workspace says");
    return ACCERL_OK;
}

LaParams la_params(const accerl_linear_attention_args* a, const LaPlan& plan) {
    LaParams p{};
    p.log_decay = a->log_decay;
    p.reset = a->reset; p.rb = a->reset_batch; p.rt = a->reset_token;
    p.lengths = a->lengths;
    p.T = a->T; p.seg_len = plan.seg_len; p.segs = plan.segs;
    p.H = a->H;
    p.groups = (uint32_t)(a->B * a->H * plan.segs);
    return p;
}
}  // namespace
}  // namespace accerl

using namespace accerl;

extern "C" {

int64_t accerl_linear_attention_workspace(int64_t B, int64_t T, int32_t H, int32_t Hk, int32_t Dk, int32_t Dv, int32_t grad) {
    if (int rc = la_check_sizes("linear_attention_workspace", B, T, H, Hk, Dk, Dv)) return rc;
    return 4 * la_work(B, T, H, Hk, Dk, Dv, grad != 0).total;
}

int accerl_linear_attention(const accerl_linear_attention_args* a, void* stream) {
    const char* who = "linear_attention";
    bool done;
    if (int rc = la_check(who, a, false, &done)) return rc;
    if (done) return ACCERL_OK;
    const int e = dtype_bytes(a->dtype);
    if (a->T > 0 && (!a->out || !la_aligned(a->out, e))) return la_fail(ACCERL_EINVAL, who, "out is NULL or misaligned");
    if (a->T > 0 && !la_spread(a->out_stride, a->B, a->T, a->H, a->Dv)) return la_fail(ACCERL_EINVAL, who, "heads of the output overlap");
    if (!la_state_ok(a->state) || !la_state_ok(a->out_state)) return la_fail(ACCERL_EINVAL, who, "states must be 16-byte aligned");
    const LaTensor out = {a->out, a->out_stride, a->H, a->Dv};
    for (const LaTensor& t : {LaTensor{a->q, a->q_stride, a->H, a->Dk}, LaTensor{a->k, a->k_stride, a->Hk, a->Dk}, LaTensor{a->v, a->v_stride, a->Hk, a->Dv}})
        if (la_overlap(out, t, a->B, a->T, e)) return la_fail(ACCERL_EINVAL, who, "out overlaps q, k or v");
    if (a->out_state != a->state && la_states_overlap(a->out_state, a->state, a)) return la_fail(ACCERL_EINVAL, who, "out_state overlaps the state other than being it");
    const LaWork k = la_work(a->B, a->T, a->H, a->Hk, a->Dk, a->Dv, false);
    if (int rc = la_workspace(who, a, k)) return rc;
    const LaParams p = la_params(a, k.plan);
    if (a->dtype == ACCERL_DT_F32) return la_forward<float>(who, *a, p, k, (float*)a->workspace, (hipStream_t)stream);
    if (a->dtype == ACCERL_DT_BF16) return la_forward<BF16>(who, *a, p, k, (float*)a->workspace, (hipStream_t)stream);
    return la_forward<F16>(who, *a, p, k, (float*)a->workspace, (hipStream_t)stream);
}

int accerl_linear_attention_grad(const accerl_linear_attention_args* a, void* stream) {
    const char* who = "linear_attention_grad";
    bool done;
    if (int rc = la_check(who, a, false, &done)) return rc;
    if (done) return ACCERL_OK;
    const int e = dtype_bytes(a->dtype);
    if (a->T > 0) {
        for (const void* p : {a->grad_out, (const void*)a->grad_q, (const void*)a->grad_k, (const void*)a->grad_v})
            if (!p || !la_aligned(p, e)) return la_fail(ACCERL_EINVAL, who, "a gradient is NULL or misaligned");
        const LaTensor in[4] = {{a->q, a->q_stride, a->H, a->Dk}, {a->k, a->k_stride, a->Hk, a->Dk}, {a->v, a->v_stride, a->Hk, a->Dv}, {a->grad_out, a->grad_out_stride, a->H, a->Dv}};
        const LaTensor to[3] = {{a->grad_q, a->grad_q_stride, a->H, a->Dk}, {a->grad_k, a->grad_k_stride, a->Hk, a->Dk}, {a->grad_v, a->grad_v_stride, a->Hk, a->Dv}};
        for (int i = 0; i < 3; ++i) {
            for (const LaTensor& t : in) if (la_overlap(to[i], t, a->B, a->T, e)) return la_fail(ACCERL_EINVAL, who, "a gradient overlaps an input");
            for (int j = 0; j < i; ++j) if (la_overlap(to[i], to[j], a->B, a->T, e)) return la_fail(ACCERL_EINVAL, who, "two gradients overlap");
        }
        if (!la_spread(a->grad_q_stride, a->B, a->T, a->H, a->Dk) || !la_spread(a->grad_k_stride, a->B, a->T, a->Hk, a->Dk) ||
            !la_spread(a->grad_v_stride, a->B, a->T, a->Hk, a->Dv)) return la_fail(ACCERL_EINVAL, who, "heads of a gradient overlap");
    }
    if (!la_state_ok(a->state) || !la_state_ok(a->grad_out_state) || !la_state_ok(a->grad_state)) return la_fail(ACCERL_EINVAL, who, "states must be 16-byte aligned");
    if (la_states_overlap(a->grad_state, a->state, a) || la_states_overlap(a->grad_state, a->grad_out_state, a)) return la_fail(ACCERL_EINVAL, who, "grad_state overlaps another state");
    const LaWork k = la_work(a->B, a->T, a->H, a->Hk, a->Dk, a->Dv, true);
    if (int rc = la_workspace(who, a, k)) return rc;
    const LaParams p = la_params(a, k.plan);
    if (a->dtype == ACCERL_DT_F32) return la_backward<float>(who, *a, p, k, (float*)a->workspace, (hipStream_t)stream);
    if (a->dtype == ACCERL_DT_BF16) return la_backward<BF16>(who, *a, p, k, (float*)a->workspace, (hipStream_t)stream);
    return la_backward<F16>(who, *a, p, k, (float*)a->workspace, (hipStream_t)stream);
}

int accerl_linear_attention_step(const accerl_linear_attention_args* a, void* stream) {
    const char* who = "linear_attention_step";
    bool done;
    if (int rc = la_check(who, a, true, &done)) return rc;
    if (done) return ACCERL_OK;
    const int e = dtype_bytes(a->dtype);
    if (!a->out || !la_aligned(a->out, e)) return la_fail(ACCERL_EINVAL, who, "out is NULL or misaligned");
    if (!la_spread({a->out_stride.batch, 0, a->out_stride.head}, a->B, 1, a->H, a->Dv)) return la_fail(ACCERL_EINVAL, who, "heads of the output overlap");
    if (!a->state || !a->out_state || !la_state_ok(a->state) || !la_state_ok(a->out_state)) return la_fail(ACCERL_EINVAL, who, "a state is NULL or not 16-byte aligned");
    if (a->out_state != a->state && la_states_overlap(a->out_state, a->state, a)) return la_fail(ACCERL_EINVAL, who, "out_state overlaps the state other than being it");
    LaStep p{};
    const int share = a->H / a->Hk;
    p.q = la_side(a->q, a->q_stride, 1); p.k = la_side(a->k, a->k_stride, share); p.v = la_side(a->v, a->v_stride, share);
    p.out = a->out; p.ob = a->out_stride.batch; p.oh = a->out_stride.head;
    p.log_decay = a->log_decay; p.reset = a->reset; p.rb = a->reset_batch;
    p.state = a->state; p.out_state = a->out_state;
    p.scale = (float)a->scale;
    p.H = a->H; p.X = a->Dk; p.Y = a->Dv; p.slices = la_slices(a->Dv);
    const hipStream_t s = (hipStream_t)stream;
    const int64_t blocks = a->B * a->H * p.slices;
    if (blocks * 256 > MAX_LAUNCH_ITEMS) return la_fail(ACCERL_EUNSUPPORTED, who, "more heads and columns than one launch takes");
    const dim3 grid((uint32_t)blocks), block(256);
    auto go = [&](auto type) {
        typedef decltype(type) T;
        if (a->Dk <= 32) la_step_kernel<T, 2><<<grid, block, 0, s>>>(p);
        else if (a->Dk <= 64) la_step_kernel<T, 4><<<grid, block, 0, s>>>(p);
        else if (a->Dk <= 128) la_step_kernel<T, 8><<<grid, block, 0, s>>>(p);
        else la_step_kernel<T, 16><<<grid, block, 0, s>>>(p);
    };
    if (a->dtype == ACCERL_DT_F32) go(0.0f);
    else if (a->dtype == ACCERL_DT_BF16) go(BF16{});
    else go(F16{});
    return la_launched(who);
}

}  // extern "C"
