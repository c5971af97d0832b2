// What the kernels share that write blocks of the paged 8-bit cache (layout: kv_common.h): conversions to codes, a block's scale, what a workgroup's wavefronts tell each other.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kv_common.h"

namespace svdq {
namespace {

__device__ __forceinline__ uint32_t max_bits_64(uint32_t m) {      // over the wavefront
    auto a = __builtin_amdgcn_permlane32_swap(m, m, false, false);
    m = a[0] > a[1] ? a[0] : a[1];
    a = __builtin_amdgcn_permlane16_swap(m, m, false, false);
    m = a[0] > a[1] ? a[0] : a[1];
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) {
        const uint32_t y = (uint32_t)__shfl_xor((int)m, o);
        m = m > y ? m : y;
    }
    return m;
}
__device__ __forceinline__ uint32_t any_bits_64(uint32_t m) {      // over the wavefront; mostly there are none
    if (__builtin_amdgcn_ballot_w64(m != 0u) == 0ull) return 0u;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m |= (uint32_t)__shfl_xor((int)m, o);
    return m;
}
__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }
__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }
constexpr uint32_t kInfBits = 0x7f800000u;

template <int N> struct RawOf;      // N 16-bit numbers as they are loaded
template <> struct RawOf<2> { typedef uint32_t type; };
template <> struct RawOf<4> { typedef uint2 type; };
template <> struct RawOf<8> { typedef uint4 type; };
typedef short short2_t __attribute__((ext_vector_type(2)));
typedef uint16_t ushort2_t __attribute__((ext_vector_type(2)));
// four numbers / 2 x 2 bf16 numbers over a power of two as four codes, round to nearest even (at most 448 of them)
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float scale) {
    short2_t w = {0, 0};
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, a, b, scale, false);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, c, d, scale, true);
    return __builtin_bit_cast(uint32_t, w);
}
__device__ __forceinline__ uint32_t codes4(uint32_t ab, uint32_t cd, float scale) {
    short2_t w = {0, 0};
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(kv_bf16x2, ab), scale, false);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(kv_bf16x2, cd), scale, true);
    return __builtin_bit_cast(uint32_t, w);
}

// The block's scale: its byte, and what codes that are in it already are multiplied by (1 if they stay).
struct BlockScale { int byte; float scale, old_factor; bool grown; };
__device__ __forceinline__ BlockScale block_scale(uint32_t amax_bits, int old_byte) {
    BlockScale s;
    const int b = kv_scale_byte(amax_bits);
    s.byte = b > old_byte ? b : old_byte;
    s.grown = s.byte > old_byte;
    s.scale = kv_pow2((s.byte < 1 ? 1 : s.byte) - 127);
    s.old_factor = kv_pow2(old_byte - s.byte < -100 ? -100 : old_byte - s.byte);
    return s;
}

// A block of a sequence: tokens lo .. hi - 1 of it are new (rows row0 + lo .. of the input), 0 .. lo - 1 are there already.
struct BlockWork { int lo, hi, blk; long long row0; };
// What a workgroup's wavefronts tell each other: tokens whose vectors are not finite, largest magnitude (bits); of keys and of values the byte that the block has.
struct Exchange { uint32_t bad[4], top[4]; int old_byte[2]; };
__device__ __forceinline__ bool live(const BlockWork &w, int tok) { return tok >= w.lo && tok < w.hi; }
__device__ __forceinline__ int readable(const BlockWork &w, int tok) { return tok < w.lo ? w.lo : tok < w.hi ? tok : w.hi - 1; }      // (a token that is not new: one that is, not used)

}  // namespace
}  // namespace svdq
