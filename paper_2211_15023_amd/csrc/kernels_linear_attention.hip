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
#include <initializer_list>
#include <type_traits>

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
    float* keep;                          // what is left of a segment's first state behind it, [segment][B H] (sums only); CUT: an episode ends in between
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

constexpr float CUT = -1.0f;
__device__ __forceinline__ float pow2(float x) { return __builtin_amdgcn_exp2f(x); }
// g^n of lg = log2 g, which may be -inf
__device__ __forceinline__ float decay_pow(float lg, int n) { return n == 0 ? 1.0f : pow2(lg * (float)n); }

// the same number of all lanes, in a scalar register
__device__ __forceinline__ float everywhere(float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); }

// How the vectors of a row are read.  EXACT: the row is as wide as the tile.  EDGE: the row has a vector at least; the last one is read so that it ends with the
// row and moved down, those behind it are zeros.  SHORT: element by element where need be.
enum LaEdge { EXACT = 0, EDGE = 1, SHORT = 2 };
// eight elements of 16 bits moved down by n (8 and more: all gone), zeros moved in
__device__ __forceinline__ u32x4 move_down(u32x4 w, int n) {
    if (n > 0) {
        if (n & 4) w = u32x4{w[2], w[3], 0, 0};
        if (n & 2) w = u32x4{w[1], w[2], w[3], 0};
        if (n & 1) w = u32x4{__builtin_amdgcn_alignbit(w[1], w[0], 16), __builtin_amdgcn_alignbit(w[2], w[1], 16), __builtin_amdgcn_alignbit(w[3], w[2], 16), w[3] >> 16};
        if (n >= 8) w = u32x4{0, 0, 0, 0};
    }
    return w;
}

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

// Which work a workgroup has.  Workgroups go round the eight XCDs: the slices of a sequence, which read the same a and b, lie eight apart.  Heads go before segments:
// those of one token lie side by side in memory (65536 tokens of 16 heads of 128, bf16: 398 us, 449 the other way round).
struct LaPlace { bool mine; uint32_t which, slice, seg, bh; };
__device__ __forceinline__ LaPlace la_place(const LaParams& p) {
    LaPlace a;
    const uint32_t id = blockIdx.x, slices = p.role[0].slices + p.role[1].slices + p.role[2].slices, grp = id / (8 * slices) * 8 + id % 8;
    a.mine = grp < p.groups;
    a.slice = id / 8 % slices;
    a.which = 0;
    while (a.slice >= (uint32_t)p.role[a.which].slices) a.slice -= p.role[a.which++].slices;
    const uint32_t heads = p.groups / p.segs;
    a.seg = grp / heads;
    a.bh = grp % heads;
    return a;
}
// A lane's part of a state: rows x + 16 ta + i, columns y0 + y + the tile's first, which is 16 d or, dealt out by fours (STEP 4), 64 (d / 4) + 4 (d % 4).
template <int STEP> __device__ __forceinline__ constexpr int la_column(int d) { return STEP == 4 ? 64 * (d / 4) + 4 * (d % 4) : STEP * d; }
template <int NA, int ND, int STEP, bool FULL>
__device__ __forceinline__ void la_state_in(const LaRole& q, uint32_t seg, uint32_t bh, int x, int y0, int y, int X, int yw, v4f (&S)[NA][ND]) {
#pragma unroll
    for (int ta = 0; ta < NA; ++ta)
#pragma unroll
        for (int d = 0; d < ND; ++d) S[ta][d] = v4f{0, 0, 0, 0};
    if (!q.enter) return;
    const float* e = q.enter + seg * q.eseg + (int64_t)bh * q.X * q.Y + x * q.ex + (y0 + y) * q.ey;
#pragma unroll
    for (int ta = 0; ta < NA; ++ta)
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if constexpr (FULL) {
                    S[ta][d][i] = e[(16 * ta + i) * q.ex + la_column<STEP>(d) * q.ey];
                } else {
                    // (those that are not there read the last one that is)
                    const int xs = min(x + 16 * ta + i, X - 1) - x, ys = min(y + la_column<STEP>(d), yw - 1) - y;
                    const float v = e[xs * q.ex + ys * q.ey];
                    S[ta][d][i] = xs == 16 * ta + i && ys == la_column<STEP>(d) ? v : 0.0f;
                }
}
template <int NA, int ND, int STEP, bool FULL>
__device__ __forceinline__ void la_state_out(const LaRole& q, uint32_t seg, uint32_t bh, int x, int y0, int y, int X, int yw, bool gone, const v4f (&S)[NA][ND]) {
    float* e = q.last + seg * q.lseg + (int64_t)bh * q.X * q.Y + x * q.lx + (y0 + y) * q.ly;
#pragma unroll
    for (int ta = 0; ta < NA; ++ta)
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (FULL || (x + 16 * ta + i < X && y + la_column<STEP>(d) < yw)) e[(16 * ta + i) * q.lx + la_column<STEP>(d) * q.ly] = gone ? 0.0f : S[ta][d][i];
}

__device__ __forceinline__ void meet() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
}
// A segment in which a NaN or an infinity was seen, in b, in c or in an output, again, token by token as the formula says: in the products a weight of 0 would carry it
// to tokens before it and to other episodes, an infinity of a would meet pairs of either sign, and a pair's product that fp32 does not hold would be an infinity though
// its weight is 0.  A lane has the rows x + 16 ta + j and columns y + la_column(d) of the state; with outputs (red) wavefront `w` of the state's leaves its part of a
// token's there, and meets those that take it.
template <typename T, int NA, int ND, int STEP, bool OUT, typename F>
__device__ __forceinline__ void la_tokens(const LaParams& p, const LaRole& q, uint32_t b, uint32_t h, int64_t n, int64_t i0, int64_t i1, float lg, int x, int y, int y0, int X, int yw,
                                          float* red, v4f (&S)[NA][ND], F taken) {
    const float ge = pow2(lg);
    const T* pa = (const T*)q.a.p + b * q.a.sb + (h / q.a.div) * q.a.sh;
    const T* pb = (const T*)q.b.p + b * q.b.sb + (h / q.b.div) * q.b.sh;
    const T* pc = (const T*)q.c.p + b * q.c.sb + (h / q.c.div) * q.c.sh + y0;
    for (int64_t i = i0; i < i1; ++i) {
        const int64_t t = q.back ? n - 1 - i : i;
        const bool anew = p.reset && (!q.back || i > 0) && p.reset[b * p.rb + (q.back ? t + 1 : t) * p.rt] != 0;
        float part[ND] = {};
#pragma unroll
        for (int ta = 0; ta < NA; ++ta)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int xx = x + 16 * ta + j;
                const float eb = xx < X ? el_f32(pb[t * q.b.st + xx]) * q.pair : 0.0f, ea = OUT && xx < X ? el_f32(pa[t * q.a.st + xx]) : 0.0f;
#pragma unroll
                for (int d = 0; d < ND; ++d) {
                    const int yy = y + la_column<STEP>(d);
                    float e = anew ? 0.0f : q.back ? S[ta][d][j] : S[ta][d][j] * ge;
                    e += eb * (yy < yw ? el_f32(pc[t * q.c.st + yy]) : 0.0f);
                    if (OUT && xx < X) part[d] += ea * e;
                    S[ta][d][j] = q.back ? e * ge : e;
                }
            }
        if constexpr (OUT) {
#pragma unroll
            for (int d = 0; d < ND; ++d) {
                part[d] += __shfl_xor(part[d], 16);
                part[d] += __shfl_xor(part[d], 32);
                if ((threadIdx.x & 63) < 16) red[y + la_column<STEP>(d)] = part[d];
            }
            meet();
            taken(i);
            meet();
        }
    }
}
// the other side of it: column y of token i from the parts of `ws` wavefronts, each LY apart
template <typename T>
__device__ __forceinline__ void la_token_out(const LaRole& q, uint32_t b, uint32_t h, int64_t n, int64_t i, int y, int y0, int yw, int ws, const float* red) {
    if (y >= yw) return;
    float v = 0.0f;
    for (int k = 0; k < ws; ++k) v += red[k * LY + y];
    v *= q.scale;
    const int64_t o = b * q.ob + (int64_t)h * q.oh + (q.back ? n - 1 - i : i) * q.ot + y0 + y;
    if (q.out_f32) ((float*)q.out)[o] = v;
    else ((T*)q.out)[o] = f32_el<T>(v);
}

// outputs of tokens behind the sequence's end
template <typename T, int NW> __device__ __forceinline__ void la_behind(const LaParams& p, const LaRole& q, const LaPlace& at, int64_t n, int64_t i0, int y0, int yw) {
    const int lane = threadIdx.x & 63;
    for (int64_t i = max(i0, n) + (threadIdx.x >> 6); i < min(p.T, i0 + p.seg_len); i += NW) {
        const int64_t o = (at.bh / p.H) * q.ob + (int64_t)(at.bh % p.H) * q.oh + i * q.ot + y0;
        for (int y = lane; y < yw; y += 64) {
            if (q.out_f32) ((float*)q.out)[o + y] = 0.0f;
            else ((T*)q.out)[o + y] = T{};
        }
    }
}

// ---------------------------------------------------------------- tokens of 16 bits
// bf16 tokens are operands as they are.  fp16 tokens are split into two bf16 parts where fp16 could not hold what they meet (weights of pairs, the state: any
// size), and the first and second order products taken: the product of both second parts, 2^-16 of a term at most, is left out, and a second part is 2^-17 off.
template <typename T, int DX, int NW>
struct LaHalf {
    static constexpr bool SPLIT = __is_same(T, F16);
    static constexpr int PARTS = SPLIT ? 2 : 1;
    // rows 16 bytes further on in the banks: a quarter wavefront's 16-byte reads of 16 rows meet no bank twice; and c's rows 8 bytes, for reads down its columns
    static constexpr int YW = 16 * NW;                        // columns of a workgroup
    static constexpr int BP = DX + 8, CP = YW + 4;
    static constexpr int NA = DX / 16 / NW, ND = NW;          // tiles of 16 rows and 16 columns of the state for a wavefront
    static constexpr int KX = DX / 32;                        // depth of the products over X in matrix instructions
    static constexpr int CT = LC * CP, SF = DX * YW, BT = LC * BP;    // elements of a tile (c: of a part) and of the state's fragments
};

__device__ __forceinline__ uint32_t high_halves(float a, float b) { return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u); }
__device__ __forceinline__ float cut16(float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); }
// a and b rounded to bf16, which are taken off them
__device__ __forceinline__ uint32_t part_pair(float& a, float& b) {
    const uint32_t p = f32_pair<BF16>(a, b);
    a -= __uint_as_float(p << 16);
    b -= __uint_as_float(p & 0xffff0000u);
    return p;
}
// Eight values as the sum of N bf16 parts.  NEAREST: each rounded, 2^-8 of the one before at most, so that two are 2^-17 off.  Else each but the second of two is cut off
// behind 8 bits, which costs less (64 x 512 tokens, 16 heads of 128, bf16: 162 us, 167 rounded; their gradients 219 and 228), and two are 2^-16 off.  Three hold all 24 bits.
template <int N, bool NEAREST> __device__ __forceinline__ void parts8(const float* x, v8bf* to) {
    u32x4 p[N];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float a = x[2 * j], b = x[2 * j + 1];
#pragma unroll
        for (int k = 0; k < N; ++k) {
            if constexpr (NEAREST) {
                p[k][j] = part_pair(a, b);
            } else {
                p[k][j] = k == 1 && N == 2 ? f32_pair<BF16>(a, b) : high_halves(a, b);
                a -= cut16(a);
                b -= cut16(b);
            }
        }
    }
#pragma unroll
    for (int k = 0; k < N; ++k) to[k] = __builtin_bit_cast(v8bf, p[k]);
}
// one part, rounded, or more
template <int N, bool NEAREST> __device__ __forceinline__ void rounded8(const float* x, v8bf* to) {
    if constexpr (N > 1) parts8<N, NEAREST>(x, to);
    else to[0] = __builtin_bit_cast(v8bf, u32x4{f32_pair<BF16>(x[0], x[1]), f32_pair<BF16>(x[2], x[3]), f32_pair<BF16>(x[4], x[5]), f32_pair<BF16>(x[6], x[7])});
}
template <typename T> __device__ __forceinline__ void unpack8(u32x4 w, float* x) {
#pragma unroll
    for (int j = 0; j < 4; ++j) el_pair<T>(w[j], x[2 * j], x[2 * j + 1]);
}
__device__ __forceinline__ v4f mma(v8bf a, v8bf b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
template <typename T> __device__ __forceinline__ v4f mma_as(u32x4 a, u32x4 b, v4f c) {
    typedef _Float16 v8h __attribute__((ext_vector_type(8)));
    if constexpr (__is_same(T, BF16)) return mma(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
}

// HOW: EXACT for heads of DX and slices of YW elements.  OUT: the mixing; else the state behind the
// segment alone.  A sequence's tokens end with a chunk, so that only the first one may be short (its tokens at its end) and the tables hold for all.
// Weights g^(63-s) of tokens s = 16 st + 4 g + i in the state behind a chunk: tail[i] block[st], neither a negative power.
struct LaTail {
    float tail[4], block[4];
    __device__ __forceinline__ LaTail(float lg, int back, float pair, int g) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            tail[i] = decay_pow(lg, 15 - 4 * g - i) * pair;
            block[i] = everywhere(decay_pow(lg, 48 - 16 * i + back));
        }
    }
};

// What NS wavefronts bring into LDS: the tiles of b and c, a chunk's tokens by DX and YW elements.
template <typename T, int DX, int YW, int NS, LaEdge HOW>
struct LaTiles {
    static constexpr bool SPLIT = __is_same(T, F16);
    static constexpr int BV = DX / 8 / NS, CV = YW / 8 / NS;                  // vectors of a lane
    static constexpr int BR = 512 * NS / DX, CR = 512 * NS / YW;              // rows from one vector of a lane to its next
    static constexpr int BP = DX + 8, CP = YW + 4;
    const LaParams& p;
    uint16_t *const sb, *const sc;
    const int bt, ct;                                         // from one tile to its twin
    const T *const pb, *const pc;                             // (SHORT) the first chunk's tiles
    const int64_t tb, tc;
    const int X, yw, gap;
    const int brow, bcol, crow, ccol, b_to, c_to;             // a lane's first vectors, and (EDGE) how far ahead they are read and to be moved from
    const T *lb, *lc;                                         // where they are in the chunk to be fetched
    const uint8_t* reset = nullptr;                           // of this lane's token there
    int64_t rt = 0, i, i0;
    int back;
    u32x4 vb[BV], vc[CV];
    uint32_t cut = 0, odd = 0;
    uint64_t cuts = 0;                                        // tokens of the staged chunk that start from nothing

    __device__ __forceinline__ LaTiles(const LaParams& p, const LaRole& q, uint16_t* sb, uint16_t* sc, int bt, int ct, const T* pb, const T* pc, int64_t tb, int64_t tc, int X, int yw, int gap,
                                       int tid)
        : p(p), sb(sb), sc(sc), bt(bt), ct(ct), pb(pb), pc(pc), tb(tb), tc(tc), X(X), yw(yw), gap(gap), brow(tid / (DX / 8)), bcol(tid % (DX / 8) * 8), crow(tid / (YW / 8)),
          ccol(tid % (YW / 8) * 8), b_to(HOW == EDGE ? min(0, X - 8 - bcol) : 0), c_to(HOW == EDGE ? min(0, yw - 8 - ccol) : 0), lb(pb + brow * tb + bcol), lc(pc + crow * tc + ccol) {}
    __device__ __forceinline__ void at(uint32_t b, int64_t n, int64_t first, int64_t base0, int backwards) {
        back = backwards;
        i = base0 + (threadIdx.x & 63);
        i0 = first;
        if (p.reset) reset = p.reset + b * p.rb + (back ? n - i : i) * p.rt;
        rt = (back ? -p.rt : p.rt) * LC;
    }
    // chunks in turn; rows of the first one that are not there count as the first that is
    template <typename F> __device__ __forceinline__ void fetch(int, F) {
        constexpr bool FIRST = F::value;
#pragma unroll
        for (int k = 0; k < BV; ++k) {
            const T* f = lb + k * BR * tb;
            if constexpr (FIRST) f += max(gap - brow - k * BR, 0) * tb;
            vb[k] = HOW == SHORT ? row_vec(bcol < X ? f : pb + gap * tb, X - bcol) : *(const u32x4_at2*)(f + b_to);
        }
#pragma unroll
        for (int k = 0; k < CV; ++k) {
            const T* f = lc + k * CR * tc;
            if constexpr (FIRST) f += max(gap - crow - k * CR, 0) * tc;
            vc[k] = HOW == SHORT ? row_vec(ccol < yw ? f : pc + gap * tc, yw - ccol) : *(const u32x4_at2*)(f + c_to);
        }
        lb += LC * tb;
        lc += LC * tc;
        // does the token of this lane start from nothing?  (backwards: does the one behind it in time)
        cut = 0;
        if (reset) {
            if (i >= i0 && !(back && i == 0)) cut = *reset;
            reset += rt;
            i += LC;
        }
    }
    template <typename F> __device__ __forceinline__ void stage(int tile, F) {
        uint16_t *const to_b = sb + tile * bt, *const to_c = sc + tile * ct;
        if constexpr (F::value) {
            const u32x4 none = {0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < BV; ++k) if (brow + k * BR < gap) vb[k] = none;
#pragma unroll
            for (int k = 0; k < CV; ++k) if (crow + k * CR < gap) vc[k] = none;
        }
        if constexpr (HOW == EDGE) {
#pragma unroll
            for (int k = 0; k < BV; ++k) vb[k] = move_down(vb[k], -b_to);
#pragma unroll
            for (int k = 0; k < CV; ++k) vc[k] = move_down(vc[k], -c_to);
        }
        typedef unsigned short us2 __attribute__((ext_vector_type(2)));
        us2 top = {0, 0};
        auto look = [&](u32x4 v) {
#pragma unroll
            for (int j = 0; j < 4; ++j) top = __builtin_elementwise_max(top, __builtin_bit_cast(us2, v[j] & 0x7fff7fffu));
        };
#pragma unroll
        for (int k = 0; k < BV; ++k) {
            look(vb[k]);
            *(u32x4*)(to_b + (brow + k * BR) * BP + bcol) = vb[k];
        }
#pragma unroll
        for (int k = 0; k < CV; ++k) {
            look(vc[k]);
            uint16_t* o = to_c + (crow + k * CR) * CP + ccol;
            if constexpr (SPLIT) {
                float x[8];
                v8bf part[2];
                unpack8<T>(vc[k], x);
                parts8<2, true>(x, part);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const u32x4 v = __builtin_bit_cast(u32x4, part[j]);
                    *(u32x2*)(o + j * LC * CP) = u32x2{v[0], v[1]};
                    *(u32x2*)(o + j * LC * CP + 4) = u32x2{v[2], v[3]};
                }
            } else {
                *(u32x2*)o = u32x2{vc[k][0], vc[k][1]};
                *(u32x2*)(o + 4) = u32x2{vc[k][2], vc[k][3]};
            }
        }
        odd |= __ballot(max((uint32_t)top[0], (uint32_t)top[1]) >= (SPLIT ? 0x7c00u : 0x7f80u)) != 0;
        cuts = __ballot(cut != 0);
    }
};

typedef __attribute__((address_space(3))) v4s la_lds4;
// Four rows of four columns each are turned by a read of 16 lanes: each has a column, down four tokens; two reads, 16 rows apart, make the eight of a fragment of 32
// tokens.
__device__ __forceinline__ u32x4 down32(const uint16_t* from, int rows16) {
    const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((la_lds4*)from), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((la_lds4*)(from + rows16));
    return __builtin_bit_cast(u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// The state behind a chunk: TERMS parts of b's weighted copy, three (without loss: it is a sum of fp32 terms) where the state is wanted.
template <typename T, typename L, int NA, int ND, int TERMS>
__device__ __forceinline__ void la_state_on(uint64_t here, float sd, LaTail& t, const uint16_t* down_b, const uint16_t* down_c, int g, v4f (&S)[NA][ND]) {
    const int last_cut = here ? 63 - __builtin_clzll(here) : -1;
    // (kept as they are: the products, worked out ahead of the loop, would take the registers)
#pragma unroll
    for (int i = 0; i < 4; ++i) asm("" : "+v"(t.tail[i]));
    if (here) {
#pragma unroll
        for (int ta = 0; ta < NA; ++ta)
#pragma unroll
            for (int d = 0; d < ND; ++d) S[ta][d] = v4f{0, 0, 0, 0};
    } else {
#pragma unroll
        for (int ta = 0; ta < NA; ++ta)
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) S[ta][d][i] *= sd;
    }
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
        float k8[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) k8[j] = t.tail[j % 4] * t.block[2 * ks + j / 4];
        if (here)
#pragma unroll
            for (int j = 0; j < 8; ++j) k8[j] = 32 * ks + (j < 4 ? 0 : 16) + 4 * g + j % 4 < last_cut ? 0.0f : k8[j];
        if constexpr (ND == 4 && TERMS == 3) {
            // (one tile of b's parts after the other: both at once, and reads ahead of them, would take the registers)
            v8bf fc[ND][L::PARTS];
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int k = 0; k < L::PARTS; ++k) fc[d][k] = __builtin_bit_cast(v8bf, down32(down_c + 32 * ks * L::CP + k * L::CT + la_column<4>(d), 16 * L::CP));
#pragma unroll
            for (int ta = 0; ta < NA; ++ta) {
                float x[8];
                v8bf fb[TERMS];
                unpack8<T>(down32(down_b + 32 * ks * L::BP + 16 * ta, 16 * L::BP), x);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] *= k8[j];
                rounded8<TERMS, L::SPLIT>(x, fb);
#pragma unroll
                for (int d = 0; d < ND; ++d) {
                    if constexpr (TERMS == 3) S[ta][d] = mma(fb[2], fc[d][0], S[ta][d]);
                    if constexpr (TERMS == 3 && L::SPLIT) S[ta][d] = mma(fb[1], fc[d][1], S[ta][d]);
                    if constexpr (TERMS >= 2) S[ta][d] = mma(fb[1], fc[d][0], S[ta][d]);
                    if constexpr (L::SPLIT) S[ta][d] = mma(fb[0], fc[d][1], S[ta][d]);
                    S[ta][d] = mma(fb[0], fc[d][0], S[ta][d]);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
            v8bf fb[NA][TERMS];
#pragma unroll
            for (int ta = 0; ta < NA; ++ta) {
                float x[8];
                unpack8<T>(down32(down_b + 32 * ks * L::BP + 16 * ta, 16 * L::BP), x);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] *= k8[j];
                rounded8<TERMS, L::SPLIT>(x, fb[ta]);
            }
#pragma unroll
            for (int d = 0; d < ND; ++d) {
                v8bf fc[L::PARTS];
#pragma unroll
                for (int k = 0; k < L::PARTS; ++k) fc[k] = __builtin_bit_cast(v8bf, down32(down_c + 32 * ks * L::CP + k * L::CT + la_column<4>(d), 16 * L::CP));
#pragma unroll
                for (int ta = 0; ta < NA; ++ta) {
                    if constexpr (TERMS == 3) S[ta][d] = mma(fb[ta][2], fc[0], S[ta][d]);
                    if constexpr (TERMS == 3 && L::SPLIT) S[ta][d] = mma(fb[ta][1], fc[1], S[ta][d]);
                    if constexpr (TERMS >= 2) S[ta][d] = mma(fb[ta][1], fc[0], S[ta][d]);
                    if constexpr (L::SPLIT) S[ta][d] = mma(fb[ta][0], fc[1], S[ta][d]);
                    S[ta][d] = mma(fb[ta][0], fc[0], S[ta][d]);
                }
            }
        }
    }
}

// The state behind a segment alone: what it adds, from nothing.  A sequence's tokens end with a chunk, so that only the first one may be short (its tokens at its
// end) and the weights hold for all.  Two of each tile: the next chunk is staged while this one is read, and a chunk has one barrier.
// b and its weight are multiplied in fp32 and handed to the matrix instructions in three bf16 parts, which hold all 24 bits: the state is as exact as in fp32.
// Bound by the splitting of b and by its chain, not by memory alone: 65536 tokens of 16 heads of 128, bf16, 137 us, 3.9 TB/s of keys and values.
// Vector instructions 53 % of the time, matrix instructions 33 %.
// HOW: EXACT for heads of DX and slices of YW elements.
template <typename T, int DX, int NW, LaEdge HOW>
__global__ __launch_bounds__(64 * NW, (LaHalf<T, DX, NW>::SPLIT || DX == 256 ? 2 : NW == 8 ? 4 : 3)) void la_sum_kernel(const LaParams p) {
    typedef LaHalf<T, DX, NW> L;
    constexpr int NA = L::NA, ND = L::ND, NB = DX == 256 ? 1 : 2;
    constexpr bool FULL = HOW == EXACT;

    __shared__ __attribute__((aligned(16))) uint16_t sb[NB * L::BT];
    __shared__ __attribute__((aligned(16))) uint16_t sc[NB * L::PARTS * L::CT];
    __shared__ int odd[NW];                                   // whether a wavefront has seen a NaN or an infinity in b or c

    const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, r = lane & 15;
    const LaPlace at = la_place(p);
    if (!at.mine) return;
    const LaRole& q = p.role[at.which];
    const int X = FULL ? DX : q.X, Y = q.Y, y0 = at.slice * L::YW, yw = FULL ? L::YW : min(Y - y0, L::YW), back = q.back;
    const uint32_t seg = at.seg, bh = at.bh, b = bh / p.H, h = bh % p.H;
    int64_t n = p.T;
    if (p.lengths) n = min(max((int64_t)p.lengths[b], (int64_t)0), n);
    const int64_t i0 = seg * p.seg_len, i1 = min(n, i0 + p.seg_len);
    const int chunks = i1 > i0 ? (int)((i1 - i0 + LC - 1) / LC) : 0;
    const int64_t base0 = i1 - (int64_t)chunks * LC;          // of the first chunk; its tokens from `gap` on are there
    const int gap = (int)(i0 - base0);
    const float lg = p.log_decay[h] * LOG2E;
    // tokens in this order: token i lies i strides behind the first
    const int64_t tb = back ? -q.b.st : q.b.st, tc = back ? -q.c.st : q.c.st, t0 = back ? n - 1 : 0;
    const T* pb = (const T*)q.b.p + b * q.b.sb + (h / q.b.div) * q.b.sh + t0 * q.b.st + base0 * tb;
    const T* pc = (const T*)q.c.p + b * q.c.sb + (h / q.c.div) * q.c.sh + t0 * q.c.st + base0 * tc + y0;
    // the state's columns, dealt out as the kernel below needs them: tile d, column r is 64 (d / 4) + 16 (r / 4) + 4 (d % 4) + r % 4
    const int yr = 16 * (r >> 2) + (r & 3);
    v4f S[NA][ND];
#pragma unroll
    for (int ta = 0; ta < NA; ++ta)
#pragma unroll
        for (int d = 0; d < ND; ++d) S[ta][d] = v4f{0, 0, 0, 0};
    LaTail tail(lg, back, q.pair, g);
    float sd = everywhere(decay_pow(lg, LC - gap)), left = 1.0f;              // (the first chunk's); what is left of a state before the segment
    bool ends = false;                                        // whether an episode does in it
    LaTiles<T, DX, L::YW, NW, HOW> tiles(p, q, sb, sc, L::BT, L::PARTS * L::CT, pb, pc, tb, tc, X, yw, gap, tid);
    tiles.at(b, n, i0, base0, back);
    const int down_b = (4 * g + (r >> 2)) * L::BP + 4 * (r & 3) + 16 * NA * w, down_c = (4 * g + (r >> 2)) * L::CP + 16 * (r & 3);
    if (chunks) {
        tiles.fetch(0, std::true_type{});
        tiles.stage(0, std::true_type{});
        if (NB == 2 && chunks > 1) tiles.fetch(1, std::false_type{});
    }
    for (int c = 0; c < chunks; ++c) {
        __syncthreads();
        const int now = NB == 2 ? c & 1 : 0;
        const uint64_t here = tiles.cuts;
        if constexpr (NB == 2) {
            if (c + 1 < chunks) {
                tiles.stage((c + 1) & 1, std::false_type{});
                if (c + 2 < chunks) tiles.fetch(c + 2, std::false_type{});
            }
        } else {
            if (c + 1 < chunks) tiles.fetch(c + 1, std::false_type{});
        }
        la_state_on<T, L, NA, ND, 3>(here, sd, tail, sb + now * L::BT + down_b, sc + now * L::PARTS * L::CT + down_c, g, S);
        left *= sd;
        ends |= here != 0;
        sd = everywhere(decay_pow(lg, LC));
        if constexpr (NB == 1) {
            __syncthreads();
            if (c + 1 < chunks) tiles.stage(0, std::false_type{});
        }
    }
    if (lane == 0) odd[w] = tiles.odd;
    __syncthreads();
    int seen = 0;
#pragma unroll
    for (int i = 0; i < NW; ++i) seen |= odd[i];
    if (seen) {
#pragma unroll
        for (int ta = 0; ta < NA; ++ta)
#pragma unroll
            for (int d = 0; d < ND; ++d) S[ta][d] = v4f{0, 0, 0, 0};
        la_tokens<T, NA, ND, 4, false>(p, q, b, h, n, i0, i1, lg, 16 * NA * w + 4 * g, yr, y0, X, yw, nullptr, S, [](int64_t) {});
    }
    // backwards the state that enters the unroll has no gradient if its first token resets
    const bool gone = back && seg == p.segs - 1 && n > 0 && p.reset && p.reset[b * p.rb] != 0;
    la_state_out<NA, ND, 4, FULL>(q, seg, bh, 16 * NA * w + 4 * g, y0, yr, X, yw, gone, S);
    if (at.slice == 0 && tid == 0) q.keep[(int64_t)seg * (p.groups / p.segs) + bh] = gone || ends ? CUT : left;
}

// The mixing itself.  Four wavefronts work out the outputs of a chunk, 16 tokens by 64 columns each, from the tiles and the state before it, while the others bring the
// state behind it and the next tiles: on every SIMD one kind's matrix instructions run beside the other's conversions, and either needs half of the registers
// that one wavefront doing both does, so that two workgroups are on a compute unit.
// A pair's product, its weight and the state's copy go into the second product as bf16, half a step each (fp16: as two bf16 parts).  64 x 512 tokens, 16 heads of 128,
// bf16, state wanted: 163 us, 4.1 TB/s of the 4.9 that a copy reaches; vector instructions 47 % of the time, matrix instructions 23 %.  What is left is a chunk's
// chain of products, barriers and state, which two workgroups a compute unit do not hide altogether.
template <typename T, int DX>
struct LaPair {
    typedef LaHalf<T, DX, 4> L;
    static constexpr int NS = DX == 256 ? 8 : 4;              // wavefronts of the state, of NA tiles of 16 rows each
    static constexpr int NA = DX / 16 / NS;
    static constexpr int THREADS = 64 * (4 + NS);
    static constexpr int WAVES = L::SPLIT ? 2 : DX == 256 ? 3 : 4;    // of a SIMD
};
// WANTED: the state behind the last token is; else b's weighted copy has two parts only, 2^-17 off, which the state's copy, rounded to one, does not show
// (gradients' states and those between segments: 65536 tokens, 16 heads of 128, bf16, 405 us; one part 397, and outputs a fifth further off).
template <typename T, int DX, LaEdge HOW, bool WANTED>
__global__ __launch_bounds__((LaPair<T, DX>::THREADS), (LaPair<T, DX>::WAVES)) void la_pair_kernel(const LaParams p) {
    typedef LaPair<T, DX> Q;
    typedef typename Q::L L;
    constexpr int NS = Q::NS, NA = Q::NA, TERMS = WANTED ? 3 : 2;
    constexpr bool FULL = HOW == EXACT;

    __shared__ __attribute__((aligned(16))) uint16_t sb[L::BT];
    __shared__ __attribute__((aligned(16))) uint16_t sc[L::PARTS * L::CT];
    // the state as the fragments that the product with a reads: [part][column tile][depth][lane][8]
    __shared__ __attribute__((aligned(16))) uint16_t ss[L::PARTS * L::SF];
    __shared__ int odd[4 + NS];                               // whether a wavefront has seen a NaN or an infinity, in an output or in b or c
    __shared__ uint64_t cut_mask;                             // tokens of the chunk that start from nothing
    __shared__ float red[NS][LY];

    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
    const LaPlace at = la_place(p);
    if (!at.mine) return;
    const LaRole& q = p.role[at.which];
    const int X = FULL ? DX : q.X, Y = q.Y, y0 = at.slice * LY, yw = FULL ? LY : min(Y - y0, LY), back = q.back;
    const uint32_t seg = at.seg, bh = at.bh, b = bh / p.H, h = bh % p.H;
    int64_t n = p.T;
    if (p.lengths) n = min(max((int64_t)p.lengths[b], (int64_t)0), n);
    const int64_t i0 = seg * p.seg_len, i1 = min(n, i0 + p.seg_len);
    const int chunks = i1 > i0 ? (int)((i1 - i0 + LC - 1) / LC) : 0;
    const int64_t base0 = i1 - (int64_t)chunks * LC;          // of the first chunk; its tokens from `gap` on are there
    const int gap = (int)(i0 - base0);
    const float lg = p.log_decay[h] * LOG2E;
    const int64_t t0 = back ? n - 1 : 0;
    const int yr = 16 * (r >> 2) + (r & 3);                   // (columns dealt out as in the sums)
    const uint16_t* down_c = sc + (4 * g + (r >> 2)) * L::CP + 16 * (r & 3);
    // at the end: has any wavefront seen a NaN or an infinity?
    auto strange = [&]() {
        int seen = 0;
#pragma unroll
        for (int i = 0; i < 4 + NS; ++i) seen |= odd[i];
        return __builtin_amdgcn_readfirstlane(seen) != 0;
    };

    if (w < 4) {
        // ------------------------------------------------ outputs
        const int64_t ta_ = back ? -q.a.st : q.a.st, to = back ? -q.ot : q.ot;
        const int t = 16 * w + r;
        const T* pa = (const T*)q.a.p + b * q.a.sb + (h / q.a.div) * q.a.sh + t0 * q.a.st + base0 * ta_;
        const T* la = pa + t * ta_ + 8 * g;
        const int64_t po = b * q.ob + (int64_t)h * q.oh + t0 * q.ot + base0 * to + y0;
        float dec[4][4];                                      // weights g^(t-s) of pairs s = 16 st + 4 g + i
#pragma unroll
        for (int st = 0; st < 4; ++st)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int s = 16 * st + 4 * g + i;
                dec[st][i] = s <= t ? decay_pow(lg, t - s) * (q.pair * q.scale) : 0.0f;
            }
        float qw = decay_pow(lg, max(t - gap, 0) + 1 - back) * q.scale;       // (the first chunk's)
        u32x4 va[L::KX];
        auto fetch_a = [&](int more) {
            const T* f = la + more * ta_;
#pragma unroll
            for (int k = 0; k < L::KX; ++k) {
                if constexpr (HOW == SHORT) va[k] = row_vec(8 * g + 32 * k < X ? f + 32 * k : f - 8 * g, X - 32 * k - 8 * g);
                else va[k] = *(const u32x4_at2*)(f + (HOW == EDGE ? min(32 * k, X - 8 - 8 * g) : 32 * k));
            }
            la += LC * ta_;
        };
        if (chunks) fetch_a(max(gap - t, 0));                 // (rows of the first chunk that are not there: the first that is)
        float zero = 0.0f;                                    // NaN from an output on that is not finite
        for (int c = 0; c < chunks; ++c) {
            meet();
            const uint64_t here = cut_mask;
            v4f O[4], P[4];
#pragma unroll
            for (int d = 0; d < 4; ++d) O[d] = P[d] = v4f{0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < L::KX; ++k) {
                v8bf fa[L::PARTS];
                if constexpr (HOW == EDGE) va[k] = move_down(va[k], max(0, 32 * k + 8 * g + 8 - X));
                if constexpr (L::SPLIT) {
                    float x[8];
                    unpack8<T>(va[k], x);
                    parts8<2, true>(x, fa);
                } else {
                    fa[0] = __builtin_bit_cast(v8bf, va[k]);
                }
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    const uint16_t* f = ss + ((d * L::KX + k) * 64 + lane) * 8;
                    if constexpr (L::SPLIT) {
                        O[d] = mma(*(const v8bf*)(f + L::SF), fa[0], O[d]);
                        O[d] = mma(*(const v8bf*)f, fa[1], O[d]);
                    }
                    O[d] = mma(*(const v8bf*)f, fa[0], O[d]);
                }
            }
            __builtin_amdgcn_sched_barrier(0);            // (reads ahead of their products would take the registers)
#pragma unroll
            for (int st = 0; st < 4; ++st)
                if (st <= w)
#pragma unroll
                    for (int k = 0; k < L::KX; ++k) P[st] = mma_as<T>(*(const u32x4*)(sb + (16 * st + r) * L::BP + 32 * k + 8 * g), va[k], P[st]);
            __builtin_amdgcn_sched_barrier(0);
            if (c + 1 < chunks) fetch_a(0);
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    O[d][i] *= qw;
                    P[d][i] *= dec[d][i];
                }
            if (here) {
                const uint64_t before = here & ((2ull << t) - 1);
                const int first = before ? 63 - __builtin_clzll(before) : -1;        // the token that t's episode begins with, if it begins in this chunk
                // (selected, not multiplied by 0: the state of the episode before may hold anything)
#pragma unroll
                for (int d = 0; d < 4; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        O[d][i] = first >= 0 ? 0.0f : O[d][i];
                        P[d][i] = 16 * d + 4 * g + i < first ? 0.0f : P[d][i];
                    }
            }
#pragma unroll
            for (int ks = 0; ks < 2; ++ks)
                if (2 * ks <= w) {
                    v8bf pt[L::PARTS];                    // weights of pairs as the product with c reads them
                    const float x[8] = {P[2 * ks][0], P[2 * ks][1], P[2 * ks][2], P[2 * ks][3], P[2 * ks + 1][0], P[2 * ks + 1][1], P[2 * ks + 1][2], P[2 * ks + 1][3]};
                    rounded8<L::PARTS, true>(x, pt);
#pragma unroll
                    for (int d = 0; d < 4; ++d) {
                        v8bf fc[L::PARTS];
#pragma unroll
                        for (int k = 0; k < L::PARTS; ++k) fc[k] = __builtin_bit_cast(v8bf, down32(down_c + 32 * ks * L::CP + k * L::CT + 4 * d, 16 * L::CP));
                        if constexpr (L::SPLIT) {
                            O[d] = mma(fc[1], pt[0], O[d]);
                            O[d] = mma(fc[0], pt[1], O[d]);
                        }
                        O[d] = mma(fc[0], pt[0], O[d]);
                    }
                }
            if (c || t >= gap) {
                const int64_t o = po + ((int64_t)c * LC + t) * to + 16 * g;
                float v[16];
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    v[j] = O[j / 4][j % 4];
                    zero = __builtin_fmaf(v[j], 0.0f, zero);
                }
                if (q.out_f32) {
                    float* f = (float*)q.out + o;
#pragma unroll
                    for (int d = 0; d < 4; ++d) {
                        if (FULL || 16 * g + 4 * d + 4 <= yw) *(u32x4_at4*)(f + 4 * d) = __builtin_bit_cast(u32x4, v4f{v[4 * d], v[4 * d + 1], v[4 * d + 2], v[4 * d + 3]});
                        else
#pragma unroll
                            for (int i = 0; i < 4; ++i) if (16 * g + 4 * d + i < yw) f[4 * d + i] = v[4 * d + i];
                    }
                } else {
                    T* f = (T*)q.out + o;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float* x = v + 8 * e;
                        if (FULL || 16 * g + 8 * e + 8 <= yw)
                            *(u32x4_at2*)(f + 8 * e) = u32x4{f32_pair<T>(x[0], x[1]), f32_pair<T>(x[2], x[3]), f32_pair<T>(x[4], x[5]), f32_pair<T>(x[6], x[7])};
                        else
#pragma unroll
                            for (int i = 0; i < 8; ++i) if (16 * g + 8 * e + i < yw) f[8 * e + i] = f32_el<T>(x[i]);
                    }
                }
            }
            qw = decay_pow(lg, t + 1 - back) * q.scale;
            meet();
        }
        const bool any = __ballot(zero != 0.0f) != 0;
        if (lane == 0) odd[w] = any;
        meet();
        if (strange())
            for (int64_t i = i0; i < i1; ++i) {
                meet();
                la_token_out<T>(q, b, h, n, i, threadIdx.x, y0, yw, NS, &red[0][0]);
                meet();
            }
        la_behind<T, 4>(p, q, at, n, i0, y0, yw);
        return;
    }

    // ---------------------------------------------------- the state and the tiles
    const int ws = w - 4, tid = threadIdx.x - 256;
    const int64_t tb = back ? -q.b.st : q.b.st, tc = back ? -q.c.st : q.c.st;
    const T* pb = (const T*)q.b.p + b * q.b.sb + (h / q.b.div) * q.b.sh + t0 * q.b.st + base0 * tb;
    const T* pc = (const T*)q.c.p + b * q.c.sb + (h / q.c.div) * q.c.sh + t0 * q.c.st + base0 * tc + y0;
    v4f S[NA][4];
    la_state_in<NA, 4, 4, FULL>(q, seg, bh, 16 * NA * ws + 4 * g, y0, yr, X, yw, S);
    LaTail tail(lg, back, q.pair, g);
    float sd = everywhere(decay_pow(lg, LC - gap));           // (the first chunk's)
    LaTiles<T, DX, LY, NS, HOW> tiles(p, q, sb, sc, 0, 0, pb, pc, tb, tc, X, yw, gap, tid);
    tiles.at(b, n, i0, base0, back);
    // the next tiles, and the state handed out
    auto hand_out = [&](auto first) {
        tiles.stage(0, first);
        if (ws == 0 && lane == 0) cut_mask = tiles.cuts;
#pragma unroll
        for (int ta = 0; ta < NA; ++ta) {
            const int tile = NA * ws + ta, quad = 4 * (tile & 1) + g;       // rows 4 quad .. of the 32 of a fragment belong to lane group quad / 2
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                uint16_t* o = ss + ((d * L::KX + (tile >> 1)) * 64 + 16 * (quad >> 1) + r) * 8 + 4 * (quad & 1);
                const v4f s = S[ta][d];
                if constexpr (L::SPLIT) {
                    float x[4] = {s[0], s[1], s[2], s[3]};
                    *(u32x2*)o = u32x2{part_pair(x[0], x[1]), part_pair(x[2], x[3])};
                    *(u32x2*)(o + L::SF) = u32x2{f32_pair<BF16>(x[0], x[1]), f32_pair<BF16>(x[2], x[3])};
                } else {
                    *(u32x2*)o = u32x2{f32_pair<BF16>(s[0], s[1]), f32_pair<BF16>(s[2], s[3])};
                }
            }
        }
    };
    const uint16_t* down_b = sb + (4 * g + (r >> 2)) * L::BP + 4 * (r & 3) + 16 * NA * ws;

    if (chunks) {
        tiles.fetch(0, std::true_type{});
        hand_out(std::true_type{});
        if (chunks > 1) tiles.fetch(1, std::false_type{});
    }
    for (int c = 0; c < chunks; ++c) {
        meet();
        la_state_on<T, L, NA, 4, TERMS>(tiles.cuts, sd, tail, down_b, down_c, g, S);
        sd = everywhere(decay_pow(lg, LC));
        meet();
        if (c + 1 < chunks) {
            hand_out(std::false_type{});
            if (c + 2 < chunks) tiles.fetch(c + 2, std::false_type{});
        }
    }
    if (lane == 0) odd[w] = tiles.odd;
    meet();
    if (strange()) {
        la_state_in<NA, 4, 4, FULL>(q, seg, bh, 16 * NA * ws + 4 * g, y0, yr, X, yw, S);
        la_tokens<T, NA, 4, 4, true>(p, q, b, h, n, i0, i1, lg, 16 * NA * ws + 4 * g, yr, y0, X, yw, red[ws], S, [](int64_t) {});
    }
    if (q.last) {
        // backwards the state that enters the unroll has no gradient if its first token resets
        const bool gone = back && seg == p.segs - 1 && n > 0 && p.reset && p.reset[b * p.rb] != 0;
        la_state_out<NA, 4, 4, FULL>(q, seg, bh, 16 * NA * ws + 4 * g, y0, yr, X, yw, gone, S);
    }
}

// ---------------------------------------------------------------- tokens of fp32
// The same walk on fp32 matrix instructions, of 32 cycles each: 304 to 448 for a wavefront and a chunk of a head of 128, at 64 columns.  32 x 512 tokens, 16 heads of 128:
// 415 us, of which matrix instructions are 38 % and vector instructions 14 %.  The rest is waiting: a comes from memory among the products of its own chunk, wavefronts
// meet whose products are uneven, and no second workgroup is on the compute unit.
template <int DX>
struct LaFloat {
    // rows 16 bytes further on in the banks, for 16-byte reads of 16 rows and for reads of four rows that lie four apart
    static constexpr int BP = DX + 4, CP = LY + 4;
    static constexpr int BV = DX / 16, CV = LY / 16;          // vectors of a lane
    static constexpr int KX = DX / 16;
};

template <int DX, bool OUT, bool FULL>
__global__ __launch_bounds__(256, DX == 64 ? 2 : 1) void la_float_kernel(const LaParams p) {
    typedef LaFloat<DX> L;
    constexpr int NA = DX / 64;                               // tiles of 16 rows of the state for a wavefront

    __shared__ __attribute__((aligned(16))) float sb[LC * L::BP];
    __shared__ __attribute__((aligned(16))) float sc[LC * L::CP];
    __shared__ __attribute__((aligned(16))) float ss[OUT ? DX * LY : 4];      // the state's fragments: [column tile][depth][lane][4]
    __shared__ int odd[4];                                    // whether a wavefront has seen a NaN or an infinity in b, c or an output
    __shared__ float red[4][LY];

    const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, r = lane & 15;
    const LaPlace at = la_place(p);
    if (!at.mine) return;
    const LaRole& q = p.role[at.which];
    const int X = FULL ? DX : q.X, Y = q.Y, y0 = at.slice * LY, yw = FULL ? LY : min(Y - y0, LY), back = q.back;
    const uint32_t seg = at.seg, bh = at.bh, b = bh / p.H, h = bh % p.H;
    int64_t n = p.T;
    if (p.lengths) n = min(max((int64_t)p.lengths[b], (int64_t)0), n);
    const int64_t i0 = seg * p.seg_len, i1 = min(n, i0 + p.seg_len);
    const int chunks = i1 > i0 ? (int)((i1 - i0 + LC - 1) / LC) : 0;
    const int64_t base0 = i1 - (int64_t)chunks * LC;          // of the first chunk; its tokens from `gap` on are there
    const int gap = (int)(i0 - base0);
    const float lg = p.log_decay[h] * LOG2E;
    const int64_t tb = back ? -q.b.st : q.b.st, tc = back ? -q.c.st : q.c.st, ta_ = back ? -q.a.st : q.a.st, to = back ? -q.ot : q.ot;
    const int64_t t0 = back ? n - 1 : 0;
    const float* pb = (const float*)q.b.p + b * q.b.sb + (h / q.b.div) * q.b.sh + t0 * q.b.st + base0 * tb;
    const float* pc = (const float*)q.c.p + b * q.c.sb + (h / q.c.div) * q.c.sh + t0 * q.c.st + base0 * tc + y0;
    const float* pa = (const float*)q.a.p + b * q.a.sb + (h / q.a.div) * q.a.sh + t0 * q.a.st + base0 * ta_;
    float* po = (float*)q.out + b * q.ob + (int64_t)h * q.oh + t0 * q.ot + base0 * to + y0;

    // the state: rows 16 (NA w + ta) + 4 g + i, columns 16 d + r
    v4f S[NA][4];
    la_state_in<NA, 4, 16, FULL>(q, seg, bh, 16 * NA * w + 4 * g, y0, r, X, yw, S);
    // weights of pairs, products of non-negative powers only: inside a tile of 16 tokens, of neighbouring tiles, of those further apart
    const int t = 16 * w + r;
    float diag[4], near[4], far[3], tail[4], block[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int s = 4 * g + i;
        diag[i] = s <= r ? decay_pow(lg, r - s) * q.pair : 0.0f;
        near[i] = decay_pow(lg, r - s + 15) * q.pair;
        tail[i] = decay_pow(lg, 15 - s) * q.pair;
        block[i] = decay_pow(lg, 48 - 16 * i + back);
    }
#pragma unroll
    for (int st = 0; st < 3; ++st) far[st] = decay_pow(lg, max(16 * (w - st) - 15, 0));
    float qw = decay_pow(lg, max(t - gap, 0) + 1 - back), sd = decay_pow(lg, LC - gap);      // (the first chunk's)
    float left = 1.0f;                                        // of the segment's first state
    bool ends = false;                                        // whether an episode does in the segment

    const int brow = tid / (DX / 4), bcol = tid % (DX / 4) * 4, crow = tid / (LY / 4), ccol = tid % (LY / 4) * 4;
    constexpr int BR = 1024 / DX, CR = 1024 / LY;             // rows from one vector of a lane to its next
    u32x4 vb[L::BV], vc[L::CV];
    uint32_t cut = 0;
    int seen = 0;                                             // a NaN or an infinity in b or c
    float zero = 0.0f;                                        // NaN from an output on that is not finite
    auto fetch = [&](int c) {
        const int skip = c ? 0 : gap;
#pragma unroll
        for (int k = 0; k < L::BV; ++k) {
            const float* f = pb + ((int64_t)c * LC + max(brow + k * BR, skip)) * tb + bcol;
            vb[k] = FULL ? *(const u32x4_at4*)f : row_vec(bcol < X ? f : pb + gap * tb, X - bcol);
        }
#pragma unroll
        for (int k = 0; k < L::CV; ++k) {
            const float* f = pc + ((int64_t)c * LC + max(crow + k * CR, skip)) * tc + ccol;
            vc[k] = FULL ? *(const u32x4_at4*)f : row_vec(ccol < yw ? f : pc + gap * tc, yw - ccol);
        }
        cut = 0;
        if (p.reset) {
            const int64_t i = base0 + (int64_t)c * LC + lane, tok = back ? n - i : i;
            if (i >= i0 && !(back && i == 0)) cut = p.reset[b * p.rb + tok * p.rt];
        }
    };
    auto stage = [&](int c) {
        uint32_t top = 0;
        const u32x4 none = {0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < L::BV; ++k) {
            if (c == 0 && brow + k * BR < gap) vb[k] = none;
#pragma unroll
            for (int j = 0; j < 4; ++j) top = max(top, vb[k][j] & 0x7fffffffu);
            *(u32x4*)(sb + (brow + k * BR) * L::BP + bcol) = vb[k];
        }
#pragma unroll
        for (int k = 0; k < L::CV; ++k) {
            if (c == 0 && crow + k * CR < gap) vc[k] = none;
#pragma unroll
            for (int j = 0; j < 4; ++j) top = max(top, vc[k][j] & 0x7fffffffu);
            *(u32x4*)(sc + (crow + k * CR) * L::CP + ccol) = vc[k];
        }
        const bool any = __ballot(top >= 0x7f800000u) != 0;
        seen |= any;
    };
    auto publish = [&]() {
        if constexpr (OUT)
#pragma unroll
            for (int ta = 0; ta < NA; ++ta)
#pragma unroll
                for (int d = 0; d < 4; ++d) *(v4f*)(ss + ((d * L::KX + NA * w + ta) * 64 + lane) * 4) = S[ta][d];
    };

    if (chunks) { fetch(0); stage(0); publish(); }
    for (int c = 0; c < chunks; ++c) {
        const uint64_t cuts = __ballot(cut != 0);
        __syncthreads();
        const bool more = c + 1 < chunks;
        // (kept as they are: their products, worked out ahead of the loop, would take 28 registers)
#pragma unroll
        for (int i = 0; i < 4; ++i) asm("" : "+v"(near[i]), "+v"(tail[i]));
        if (more) fetch(c + 1);
        const int last_cut = cuts ? 63 - __builtin_clzll(cuts) : -1;

        v4f O[4];
        float wt[4][4];
        if constexpr (OUT) {
            const float* ra = pa + ((int64_t)c * LC + max(t, c ? 0 : gap)) * ta_ + 4 * g;
            v4f P[4];
#pragma unroll
            for (int st = 0; st < 4; ++st) O[st] = P[st] = v4f{0, 0, 0, 0};
#pragma unroll 4
            for (int k = 0; k < L::KX; ++k) {
                const v4f fa = __builtin_bit_cast(v4f, FULL ? *(const u32x4_at4*)(ra + 16 * k) : row_vec(4 * g + 16 * k < X ? ra + 16 * k : ra - 4 * g, X - 16 * k - 4 * g));
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
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) O[d][i] *= qw;
#pragma unroll
            for (int st = 0; st < 4; ++st) {
#pragma unroll
                for (int i = 0; i < 4; ++i) wt[st][i] = 0.0f;
                if (st == w) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) wt[st][i] = P[st][i] * diag[i];
                } else if (st < w) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) wt[st][i] = P[st][i] * (near[i] * far[st < 3 ? st : 0]);
                }
            }
            if (cuts) {
                const uint64_t before = cuts & ((2ull << t) - 1);
                const int first = before ? 63 - __builtin_clzll(before) : -1;        // the token that t's episode begins with, if it begins in this chunk
                // (selected, not multiplied by 0: the state of the episode before may hold anything)
                if (first >= 0)
#pragma unroll
                    for (int d = 0; d < 4; ++d) O[d] = v4f{0, 0, 0, 0};
#pragma unroll
                for (int st = 0; st < 4; ++st)
#pragma unroll
                    for (int i = 0; i < 4; ++i) if (16 * st + 4 * g + i < first) wt[st][i] = 0.0f;
            }
        }
        // what enters the next chunk
#pragma unroll
        for (int ta = 0; ta < NA; ++ta)
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) S[ta][d][i] = cuts ? 0.0f : S[ta][d][i] * sd;
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
                    for (int i = 0; i < 4; ++i) O[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(fc[d][i], wt[st][i], O[d], 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int s = 16 * st + 4 * g + i;
                const float kw = s < last_cut ? 0.0f : tail[i] * block[st];
#pragma unroll
                for (int ta = 0; ta < NA; ++ta) {
                    const float x = sb[s * L::BP + 16 * (NA * w + ta) + r] * kw;
#pragma unroll
                    for (int d = 0; d < 4; ++d) S[ta][d] = __builtin_amdgcn_mfma_f32_16x16x4f32(x, fc[d][i], S[ta][d], 0, 0, 0);
                }
            }
        }
        if constexpr (OUT) {
            if (c || t >= gap) {
                float* f = po + ((int64_t)c * LC + t) * to;
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    const int y = 16 * d + 4 * g;
                    v4f v = O[d];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        v[i] *= q.scale;
                        zero = __builtin_fmaf(v[i], 0.0f, zero);
                    }
                    if (FULL || y + 4 <= yw) *(u32x4_at4*)(f + y) = __builtin_bit_cast(u32x4, v);
                    else
#pragma unroll
                        for (int i = 0; i < 4; ++i) if (y + i < yw) f[y + i] = v[i];
                }
            }
        }

        left *= sd;
        ends |= cuts != 0;
        qw = decay_pow(lg, t + 1 - back);
        sd = decay_pow(lg, LC);
        __syncthreads();
        if (more) { stage(c + 1); publish(); }
    }

    if constexpr (OUT) {
        const bool any = __ballot(zero != 0.0f) != 0;
        seen |= any;
    }
    if (lane == 0) odd[w] = seen;
    __syncthreads();
    if (odd[0] | odd[1] | odd[2] | odd[3]) {
        if constexpr (OUT) la_state_in<NA, 4, 16, FULL>(q, seg, bh, 16 * NA * w + 4 * g, y0, r, X, yw, S);
        else
#pragma unroll
            for (int ta = 0; ta < NA; ++ta)
#pragma unroll
                for (int d = 0; d < 4; ++d) S[ta][d] = v4f{0, 0, 0, 0};
        la_tokens<float, NA, 4, 16, OUT>(p, q, b, h, n, i0, i1, lg, 16 * NA * w + 4 * g, r, y0, X, yw, red[w], S,
                                         [&](int64_t i) { la_token_out<float>(q, b, h, n, i, tid, y0, yw, 4, &red[0][0]); });
    }
    if (q.last) {
        const bool gone = back && seg == p.segs - 1 && n > 0 && p.reset && p.reset[b * p.rb] != 0;
        la_state_out<NA, 4, 16, FULL>(q, seg, bh, 16 * NA * w + 4 * g, y0, r, X, yw, gone, S);
        if (q.keep && at.slice == 0 && tid == 0) q.keep[(int64_t)seg * (p.groups / p.segs) + bh] = gone || ends ? CUT : left;
    }
    if constexpr (OUT) la_behind<float, 4>(p, q, at, n, i0, y0, yw);
}

// The states that enter the segments, from what each segment adds: states [segment][B H][X Y] in place, the last one to `last`.
// Bound by memory and by the chain of the segments (64 segments of 16 heads of 128 x 128: 12 us for 67 MB read and written).
struct LaJoin { float* states; const float* keep; const float* enter; float* last; };
struct LaJoinParams { LaJoin at[2]; const float* log_decay; int64_t n, per; int H, segs; };     // n = B H X Y, per = X Y
__global__ __launch_bounds__(256) void la_join_kernel(const LaJoinParams p) {
    const LaJoin& j = p.at[blockIdx.y];
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= p.n) return;
    const int64_t bh = i / p.per, all = p.n / p.per;
    float e = j.enter ? j.enter[i] : 0.0f;
    // (an infinity stays one under any decay but 0, which makes it NaN, also where the power is 0 in fp32)
    const float stays = p.log_decay[bh % p.H] == -INFINITY ? 0.0f : 1.0f;
    constexpr int AT_ONCE = 8;                                // loads under way together
    for (int s0 = 0; s0 < p.segs; s0 += AT_ONCE) {
        float add[AT_ONCE], f[AT_ONCE];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const int s = min(s0 + k, p.segs - 1);
            add[k] = j.states[s * p.n + i];
            f[k] = j.keep[s * all + bh];
        }
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k)
            if (s0 + k < p.segs) {
                j.states[(s0 + k) * p.n + i] = e;
                const float on = f[k] > 0.0f ? f[k] * e : isfinite(e) ? 0.0f : e * stays;
                e = (f[k] == CUT ? 0.0f : on) + add[k];
            }
    }
    if (j.last) j.last[i] = e;
}

// The gradients of shared keys and values: the heads' parts [B, T, H, D] in fp32, summed in the heads' order and rounded once.
// Bound by memory, or a launch (5 x 333 tokens: 4 us).
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
// is read and written once.  FULL: 16 ROWS rows, and columns in whole workgroups.  ONCE: states that are more than the caches hold go by them.
// 512 environments of 16 heads of 128, bf16 tokens: 190 us, 5.7 TB/s.
template <typename T, int ROWS, bool FULL, bool ONCE>
__global__ __launch_bounds__(256, ROWS <= 4 ? 8 : ROWS == 8 ? 6 : 4) void la_step_kernel(const LaStep p) {
    __shared__ v4f red[4][16];
    const int tid = threadIdx.x, w = tid >> 6, lane = tid & 63, r = lane & 15, x0 = tid >> 4;
    const uint32_t slice = blockIdx.x % p.slices, bh = blockIdx.x / p.slices, b = bh / p.H, h = bh % p.H;
    const int y = slice * 64 + 4 * r, in = FULL ? 4 : min(max(p.Y - y, 0), 4), X = FULL ? 16 * ROWS : p.X;
    const bool anew = p.reset && p.reset[b * p.rb] != 0;
    const T* pq = (const T*)p.q.p + b * p.q.sb + h * p.q.sh + x0;
    const T* pk = (const T*)p.k.p + b * p.k.sb + (h / p.k.div) * p.k.sh + x0;
    const T* pv = (const T*)p.v.p + b * p.v.sb + (h / p.v.div) * p.v.sh + (in ? y : 0);
    const int64_t at = (int64_t)bh * X * p.Y + (int64_t)x0 * p.Y + (in ? y : 0);
    const float* s = p.state + at;
    float* so = p.out_state + at;
    const int rows16 = 16 * p.Y;
    v4f S[ROWS];
    T k[ROWS], q[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        S[i] = v4f{0, 0, 0, 0};
        if (!anew && (FULL || x0 + 16 * i < X)) {
            if constexpr (FULL && ONCE) S[i] = __builtin_nontemporal_load((const v4f*)(s + i * rows16));
            else if constexpr (FULL) S[i] = *(const v4f*)(s + i * rows16);
            else S[i] = __builtin_bit_cast(v4f, row_vec(s + i * rows16, in));
        }
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const bool there = FULL || x0 + 16 * i < X;
        k[i] = there ? pk[16 * i] : T{};
        q[i] = there ? pq[16 * i] : T{};
    }
    v4f v = {0, 0, 0, 0}, o = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < 4; ++j) if (j < in) v[j] = el_f32(pv[j]);
    const float ge = anew ? 0.0f : pow2(p.log_decay[h] * LOG2E);
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const float kx = el_f32(k[i]), qx = el_f32(q[i]);
#pragma unroll
        for (int j = 0; j < 4; ++j) S[i][j] = ge * S[i][j] + kx * v[j];
        // (a row that is not there has no part in the output: an infinity of v times its key of 0 would be NaN)
        if (FULL || x0 + 16 * i < X) {
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] += qx * S[i][j];
            if constexpr (FULL && ONCE) __builtin_nontemporal_store(S[i], (v4f*)(so + i * rows16));
            else if (in == 4) *(u32x4_at4*)(so + i * rows16) = __builtin_bit_cast(u32x4, S[i]);
            else
#pragma unroll
                for (int j = 0; j < 4; ++j) if (j < in) so[i * rows16 + j] = S[i][j];
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
// What the caches hold.  One token's states of 16 heads of 128, read and written: 192 MB 61 us, and 70 by the caches; 512 MB 208 us, and 189 by the caches.
constexpr int64_t ONCE_BYTES = 256 << 20;
// From here on the segments' sums take 128 columns a workgroup, which read b half as often (65536 tokens, 16 heads of 128, bf16: 405 us in all, a sixteenth more with 64 columns).
constexpr uint32_t WIDE_GROUPS = 512;
// Up to here the gradients' roles of two widths share a launch (2 x 200 tokens, 4 heads of 48 and 72, bf16: 20 us, 28 one by one); with more the padding costs more
// (8 x 256 tokens, 8 heads of 100 and 200, fp32: 202 us, 166 one by one).
constexpr int64_t TOGETHER_BLOCKS = 256;
struct LaPlan { int segs; int64_t seg_len; };
// Segments of a sequence, worked on side by side, where sequences, heads and columns alone leave compute units without work: what each adds to the state is summed
// first, so keys and values are read twice, and states go through memory.  From how many chunks on that pays, by workgroups without it:
//     heads of 128, us whole / in segments     8: 3 chunks, 8, 16          64: 8 chunks, 16, 32          128: 16 chunks, 64        256: 64 chunks
//     bf16                                     11/16, 20/17, 36/20         22/32, 37/37, 69/45           39/46, 139/118            156/221
//     fp16                                     14/17, 30/19, 55/22         31/38, 56/46, 107/63          57/65, 212/193            231/341
//     fp32 (bound by its chain)                33/25, 81/26, 157/29        84/53, 174/80, 343/135        175/136, 765/519          777/990
LaPlan la_plan(int64_t B, int64_t T, int H, int slices, bool f32) {
    const int64_t blocks = B * H * slices, chunks = (T + LC - 1) / LC;
    int64_t segs = 1;
    if (blocks > 0 && (f32 ? blocks < 192 && chunks >= std::max<int64_t>(3, blocks / 16) : blocks < 160 && chunks >= std::max<int64_t>(8, blocks * blocks / 256))) {
        // as many as are on the chip at once; twice as many where each still has eight chunks (65536 tokens, 16 heads of 128, bf16: 398 us with 1024, 420 with 512,
        // 425 with 2048; 3 x 1777 tokens, 6 heads of 80 and 100, fp16: 49 us with 512, 65 with 1024)
        const int64_t most = blocks * chunks >= 8 * 1024 ? 1024 : 512;
        segs = std::max<int64_t>(1, std::min<int64_t>((most + blocks - 1) / blocks, chunks));
    }
    const int64_t per = std::max<int64_t>(1, (chunks + segs - 1) / segs);
    return {(int)std::max<int64_t>(1, (chunks + per - 1) / per), per * LC};
}
int la_slices(int y) { return (y + LY - 1) / LY; }
int64_t la_up(int64_t n) { return (n + 15) / 16 * 16; }

// floats of the workspace: the segments' states and what each keeps, for the state and (gradients) its gradient; the parts of shared gradients
struct LaWork { LaPlan plan; int64_t states, keep, parts_k, parts_v, total; };
LaWork la_work(int64_t B, int64_t T, int H, int Hk, int Dk, int Dv, bool grad, bool f32) {
    LaWork k{};
    k.plan = la_plan(B, T, H, grad ? 2 * la_slices(Dk) + la_slices(Dv) : la_slices(Dv), f32);
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

template <typename T, int DX, bool OUT>
void la_go(const LaParams& p, bool wide, LaEdge how, bool wanted, dim3 grid, hipStream_t s) {
    auto go = [&](auto kind) {
        constexpr LaEdge HOW = decltype(kind)::value;
        if constexpr (__is_same(T, float)) la_float_kernel<DX, OUT, HOW == EXACT><<<grid, dim3(256), 0, s>>>(p);
        else if constexpr (OUT) {
            const dim3 block(LaPair<T, DX>::THREADS);
            if (wanted) la_pair_kernel<T, DX, HOW, true><<<grid, block, 0, s>>>(p);
            else la_pair_kernel<T, DX, HOW, false><<<grid, block, 0, s>>>(p);
        } else {
            if constexpr (DX > 64) if (wide) return la_sum_kernel<T, DX, 8, HOW><<<grid, dim3(512), 0, s>>>(p);
            la_sum_kernel<T, DX, 4, HOW><<<grid, dim3(256), 0, s>>>(p);
        }
    };
    if (how == EXACT) go(std::integral_constant<LaEdge, EXACT>());
    else if (how == EDGE || __is_same(T, float)) go(std::integral_constant<LaEdge, EDGE>());
    else go(std::integral_constant<LaEdge, SHORT>());
}
template <typename T, bool OUT>
int la_launch(const char* who, LaParams p, int X, hipStream_t s) {
    // (the segments' sums: fewer and wider workgroups where there are enough of them to go round)
    int slices = 0, most = 0, least = LA_MAX_D;
    for (const LaRole& r : p.role)
        if (r.slices) {
            most = std::max(most, r.Y);
            least = std::min(least, std::min(r.X, r.Y));
        }
    const bool wide = !OUT && !__is_same(T, float) && X > 64 && most > LY && least >= 8 && p.groups >= WIDE_GROUPS;
    const int cols = wide ? 2 * LY : LY;
    LaEdge how = least < 8 ? SHORT : EXACT;
    bool wanted = false;
    for (LaRole& r : p.role) {
        if (!r.slices) continue;
        if (r.last) wanted = true;
        r.slices = (r.Y + cols - 1) / cols;
        slices += r.slices;
        if (how == EXACT && (r.X != X || r.Y % cols)) how = EDGE;
    }
    const int64_t blocks = ((int64_t)p.groups + 7) / 8 * 8 * slices;
    const dim3 grid((uint32_t)blocks);
    if (X == 64) la_go<T, 64, OUT>(p, wide, how, wanted, grid, s);
    else if (X == 128) la_go<T, 128, OUT>(p, wide, how, wanted, grid, s);
    else la_go<T, 256, OUT>(p, wide, how, wanted, grid, s);
    return la_launched(who);
}
int la_pad(int x) { return x <= 64 ? 64 : x <= 128 ? 128 : 256; }

// Launches of the roles, those of one width together (gradients of 32 x 512 tokens, 16 heads of 128, bf16: 219 us, 227 with those whose state is not wanted in a launch of
// their own), and all in the widest one's where they leave compute units without work one by one.
template <typename T, bool OUT>
int la_run(const char* who, const LaParams& common, const LaRole* roles, int count, hipStream_t s) {
    int64_t blocks = 0;
    int widest = 0;
    for (int i = 0; i < count; ++i) {
        blocks += (int64_t)common.groups * roles[i].slices;
        widest = std::max(widest, la_pad(roles[i].X));
    }
    const bool together = blocks <= TOGETHER_BLOCKS;
    // (all of them with the widest workgroup's threads, groups rounded up to eight: nothing is enqueued of a call that a later launch would refuse)
    if ((blocks + 8 * 12) * 768 > MAX_LAUNCH_ITEMS) return la_fail(ACCERL_EUNSUPPORTED, who, "more heads, segments and columns than one launch takes");
    for (int x : {64, 128, 256}) {
        LaParams p = common;
        int n = 0;
        for (int i = 0; i < count; ++i) if ((together ? widest : la_pad(roles[i].X)) == x) p.role[n++] = roles[i];
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
        j.log_decay = p.log_decay; j.n = n; j.per = per; j.H = p.H; j.segs = p.segs;
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

int64_t la_fold_items(const accerl_linear_attention_args& a) { return a.B * a.T * a.Hk * (int64_t)std::max(a.Dk, a.Dv); }
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
        j.log_decay = p.log_decay; j.n = n; j.per = per; j.H = p.H; j.segs = p.segs;
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
    if (share > 1 && a.T > 0) {                               // (no launch is of nothing)
        LaFoldParams f{};
        f.at[0] = {parts_k, a.grad_k, a.grad_k_stride.batch, a.grad_k_stride.token, a.grad_k_stride.head, a.Dk};
        f.at[1] = {parts_v, a.grad_v, a.grad_v_stride.batch, a.grad_v_stride.token, a.grad_v_stride.head, a.Dv};
        f.tokens = a.B * a.T; f.T = a.T; f.H = a.H; f.Hk = a.Hk;
        la_fold_kernel<T><<<dim3((uint32_t)((la_fold_items(a) + 255) / 256), 2), dim3(256), 0, s>>>(f);
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

// What a call reads and writes, as runs of bytes.
Strided la_tokens_at(const accerl_linear_attention_args& a, const void* p, const accerl_token_stride& s, int H, int D, int64_t T) {
    const int64_t e = dtype_bytes(a.dtype);
    return Strided(p, a.B, s.batch * e, T, s.token * e, H, s.head * e, D * e);
}
Strided la_states_at(const accerl_linear_attention_args& a, const void* p) { return Strided(p, 4 * a.B * a.H * a.Dk * a.Dv); }
struct LaInputs {
    Strided q, k, v, log_decay, reset, lengths, state;
    LaInputs(const accerl_linear_attention_args& a, int64_t T, const int32_t* lengths)
        : q(la_tokens_at(a, a.q, a.q_stride, a.H, a.Dk, T)), k(la_tokens_at(a, a.k, a.k_stride, a.Hk, a.Dk, T)), v(la_tokens_at(a, a.v, a.v_stride, a.Hk, a.Dv, T)),
          log_decay(a.log_decay, 4 * (int64_t)a.H), reset(a.reset, a.B, a.reset_batch, T, a.reset_token, 1, 0, 1), lengths(lengths, 4 * a.B), state(la_states_at(a, a.state)) {}
};
typedef std::initializer_list<const Strided*> LaList;
bool la_any_share(LaList outs, LaList others) {
    for (const Strided* o : outs)
        for (const Strided* t : others) if (share(*o, *t)) return true;
    return false;
}
// an unroll's or a step's outputs; out_state may be the state
int la_outputs_apart(const char* who, const accerl_linear_attention_args* a, const LaInputs& in, const Strided& out, const Strided& out_state) {
    if (la_any_share({&out, &out_state}, {&in.q, &in.k, &in.v, &in.log_decay, &in.reset, &in.lengths})) return la_fail(ACCERL_EINVAL, who, "an output overlaps an input");
    if (la_any_share({&out}, {&in.state, &out_state})) return la_fail(ACCERL_EINVAL, who, "out overlaps a state");
    if (a->out_state != a->state && share(out_state, in.state)) return la_fail(ACCERL_EINVAL, who, "out_state overlaps the state other than being it");
    return ACCERL_OK;
}

int la_workspace(const char* who, const accerl_linear_attention_args* a, const LaWork& k, LaList all) {
    if (k.total == 0) return ACCERL_OK;
    if (!a->workspace || !la_aligned(a->workspace, 16)) return la_fail(ACCERL_EINVAL, who, "workspace is NULL or misaligned");
    if (a->workspace_bytes < 4 * k.total) return la_fail(ACCERL_EINVAL, who, "workspace smaller than accerl_linear_attention_workspace says");
    const Strided work(a->workspace, 4 * k.total);
    if (la_any_share({&work}, all)) return la_fail(ACCERL_EINVAL, who, "the workspace overlaps an input or an output");
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
    // (of either kind of tokens)
    return 4 * std::max(la_work(B, T, H, Hk, Dk, Dv, grad != 0, false).total, la_work(B, T, H, Hk, Dk, Dv, grad != 0, true).total);
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
    const LaInputs in(*a, a->T, a->lengths);
    const Strided out = la_tokens_at(*a, a->out, a->out_stride, a->H, a->Dv, a->T), out_state = la_states_at(*a, a->out_state);
    if (int rc = la_outputs_apart(who, a, in, out, out_state)) return rc;
    const LaWork k = la_work(a->B, a->T, a->H, a->Hk, a->Dk, a->Dv, false, a->dtype == ACCERL_DT_F32);
    if (int rc = la_workspace(who, a, k, {&in.q, &in.k, &in.v, &in.log_decay, &in.reset, &in.lengths, &in.state, &out, &out_state})) return rc;
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
        if (!la_spread(a->grad_q_stride, a->B, a->T, a->H, a->Dk) || !la_spread(a->grad_k_stride, a->B, a->T, a->Hk, a->Dk) ||
            !la_spread(a->grad_v_stride, a->B, a->T, a->Hk, a->Dv)) return la_fail(ACCERL_EINVAL, who, "heads of a gradient overlap");
    }
    if (!la_state_ok(a->state) || !la_state_ok(a->grad_out_state) || !la_state_ok(a->grad_state)) return la_fail(ACCERL_EINVAL, who, "states must be 16-byte aligned");
    if (a->H != a->Hk && la_fold_items(*a) > MAX_LAUNCH_ITEMS - 256) return la_fail(ACCERL_EUNSUPPORTED, who, "more gradients of shared heads than one launch takes");
    const LaInputs in(*a, a->T, a->lengths);
    const Strided go = la_tokens_at(*a, a->grad_out, a->grad_out_stride, a->H, a->Dv, a->T), gs = la_states_at(*a, a->grad_out_state);
    const Strided gq = la_tokens_at(*a, a->grad_q, a->grad_q_stride, a->H, a->Dk, a->T), gk = la_tokens_at(*a, a->grad_k, a->grad_k_stride, a->Hk, a->Dk, a->T);
    const Strided gv = la_tokens_at(*a, a->grad_v, a->grad_v_stride, a->Hk, a->Dv, a->T), gstate = la_states_at(*a, a->grad_state);
    if (la_any_share({&gq, &gk, &gv, &gstate}, {&in.q, &in.k, &in.v, &go, &in.log_decay, &in.reset, &in.lengths, &in.state, &gs}))
        return la_fail(ACCERL_EINVAL, who, "a gradient overlaps an input");
    if (la_any_share({&gq}, {&gk, &gv, &gstate}) || la_any_share({&gk}, {&gv, &gstate}) || share(gv, gstate)) return la_fail(ACCERL_EINVAL, who, "two gradients overlap");
    const LaWork k = la_work(a->B, a->T, a->H, a->Hk, a->Dk, a->Dv, true, a->dtype == ACCERL_DT_F32);
    if (int rc = la_workspace(who, a, k, {&in.q, &in.k, &in.v, &go, &in.log_decay, &in.reset, &in.lengths, &in.state, &gs, &gq, &gk, &gv, &gstate})) return rc;
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
    if (int rc = la_outputs_apart(who, a, LaInputs(*a, 1, nullptr), la_tokens_at(*a, a->out, a->out_stride, a->H, a->Dv, 1), la_states_at(*a, a->out_state))) return rc;
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
    const bool whole = a->Dv % 64 == 0, once = 4 * a->B * a->H * (int64_t)a->Dk * a->Dv > ONCE_BYTES;
    auto go = [&](auto type) {
        typedef decltype(type) T;
        auto rows = [&](auto n) {
            constexpr int ROWS = decltype(n)::value;
            if (!(whole && a->Dk == 16 * ROWS)) la_step_kernel<T, ROWS, false, false><<<grid, block, 0, s>>>(p);
            else if (once) la_step_kernel<T, ROWS, true, true><<<grid, block, 0, s>>>(p);
            else la_step_kernel<T, ROWS, true, false><<<grid, block, 0, s>>>(p);
        };
        if (a->Dk <= 32) rows(std::integral_constant<int, 2>());
        else if (a->Dk <= 64) rows(std::integral_constant<int, 4>());
        else if (a->Dk <= 128) rows(std::integral_constant<int, 8>());
        else rows(std::integral_constant<int, 16>());
    };
    if (a->dtype == ACCERL_DT_F32) go(0.0f);
    else if (a->dtype == ACCERL_DT_BF16) go(BF16{});
    else go(F16{});
    return la_launched(who);
}

}  // extern "C"
