// What the operators of wide policies share: element types and their conversions, loads of any alignment.
#pragma once
#include "accerl_internal.h"
#include "tables.h"

namespace accerl {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
// rows may start anywhere (odd widths): these vectors are aligned to one element only, which a vector load or store of the device takes
typedef u32x4 u32x4_at4 __attribute__((aligned(4)));
typedef u32x4 u32x4_at2 __attribute__((aligned(2)));
typedef u32x2 u32x2_at2 __attribute__((aligned(2)));

struct BF16 { uint16_t u; };
struct F16 { uint16_t u; };

inline int dtype_bytes(int dtype) { return dtype == ACCERL_DT_F32 ? 4 : 2; }
inline bool dtype_known(int dtype) { return dtype == ACCERL_DT_F32 || dtype == ACCERL_DT_BF16 || dtype == ACCERL_DT_F16; }

__device__ __forceinline__ float el_f32(float x) { return x; }
__device__ __forceinline__ float el_f32(BF16 x) { return __uint_as_float((uint32_t)x.u << 16); }
__device__ __forceinline__ float el_f32(F16 x) { _Float16 h; __builtin_memcpy(&h, &x, 2); return (float)h; }

// the two elements of a 32-bit word
template <typename T> __device__ __forceinline__ void el_pair(uint32_t w, float& a, float& b) {
    if constexpr (__is_same(T, BF16)) { a = __uint_as_float(w << 16); b = __uint_as_float(w & 0xffff0000u); }
    else { typedef _Float16 h2 __attribute__((ext_vector_type(2))); const h2 h = __builtin_bit_cast(h2, w); a = (float)h[0]; b = (float)h[1]; }
}
// rounded to nearest even, infinities and NaN kept
template <typename T> __device__ __forceinline__ T f32_el(float x) {
    if constexpr (__is_same(T, float)) return x;
    else if constexpr (__is_same(T, BF16)) { const __bf16 b = (__bf16)x; return __builtin_bit_cast(BF16, b); }
    else { const _Float16 h = (_Float16)x; return __builtin_bit_cast(F16, h); }
}
template <typename T> __device__ __forceinline__ uint32_t f32_pair(float a, float b) {
    if constexpr (__is_same(T, BF16)) {
        typedef __bf16 b2 __attribute__((ext_vector_type(2)));
        const b2 v = {(__bf16)a, (__bf16)b};
        return __builtin_bit_cast(uint32_t, v);
    } else {
        typedef _Float16 h2 __attribute__((ext_vector_type(2)));
        const h2 v = {(_Float16)a, (_Float16)b};
        return __builtin_bit_cast(uint32_t, v);
    }
}

}  // namespace accerl
