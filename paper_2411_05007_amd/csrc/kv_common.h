// What the kernels of the paged 8-bit cache of keys and values share: the cache's layout, the work items of a ragged batch, the
// position rotation, the conversions to and from E4M3 codes.
//
// A cache has pages of P tokens (32 to 1024, a power of two), cut into blocks of 32 tokens, and a scale byte for each block and head
// (value 2^(byte - 127), 0: a block of zeros), keys and values apart.  The codes of one block and head are 32 D bytes in a row:
//   keys    [32][D]: a row of a block is the operand row of K Q^T as it lies
//   values  [D / 32][16][4][2][8], transposed: element (t, d) at [d / 32][d % 16][g][(d % 32) / 16][j], slot g = 2 (t / 16) + (t % 8) / 4,
//           j = 4 ((t % 16) / 8) + t % 4.  The accumulators of S^T = K Q^T on 32 x 32 blocks hold the tokens of slots 2 s + h, s = 0, 1, in lane
//           half h, eight in the order of j: they are the operand of O^T = V^T P^T with no exchange between lanes.
// Why E4M3 with powers of two: gfx950 turns two codes and a power of two into two exact f16 (or bf16) numbers in one instruction; a
// power of two can grow while its block fills without a second rounding of the normal codes that are in it; and what a score owes to
// its block's scale is one factor for 32 tokens.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.h"

namespace svdq {

constexpr int kKvBlock = 32;                     // tokens with one scale
constexpr uint32_t kKvNaN = 0x7fu;               // the NaN code

typedef _Float16 kv_f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 kv_f16x8 __attribute__((ext_vector_type(8)));
typedef float kv_floatx2 __attribute__((ext_vector_type(2)));
typedef float kv_floatx4 __attribute__((ext_vector_type(4)));
typedef float kv_floatx16 __attribute__((ext_vector_type(16)));
typedef __bf16 kv_bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t kv_u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t kv_u32x2 __attribute__((ext_vector_type(2)));

// tokens of slot g: kv_slot_token(g) + {0, 1, 2, 3, 8, 9, 10, 11}
__host__ __device__ constexpr int kv_slot_token(int g) { return 16 * (g >> 1) + 4 * (g & 1); }

// ---- work items of a ragged batch -----------------------------------------------------------------------------------------
// The sequences' items lie behind each other: a workgroup finds its own by a scan over how many each sequence has, 64 sequences a round, from lengths
// that the host need not know; a grid of more items than there are is empty at its end only.  (With room for every sequence's remainder behind its own items, every other
// workgroup of equal short sequences was empty, the dispatcher put the others on half of the CUs, and 32 sequences of 128 rows on 4128 keys took 259 us instead of 162.)
// cu is taken within 0 .. T, as far as it ascends.
struct KvItem { int sequence, local, first, count, value; };      // local: which item of the sequence, -1: none; its tokens; kv_len as it stands
__device__ __forceinline__ int kv_within(int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; }
// sum over the lanes up to this one
template <int CONTROL, int ROWS>
__device__ __forceinline__ int kv_add_dpp(int x) { return x + __builtin_amdgcn_update_dpp(0, x, CONTROL, ROWS, 0xf, true); }
__device__ __forceinline__ int kv_sum_upto(int x) {
    x = kv_add_dpp<0x118, 0xf>(kv_add_dpp<0x114, 0xf>(kv_add_dpp<0x112, 0xf>(kv_add_dpp<0x111, 0xf>(x))));      // within sixteen lanes: from 1, 2, 4, 8 lanes below
    return kv_add_dpp<0x143, 0xc>(kv_add_dpp<0x142, 0xa>(x));      // the second and fourth sixteen take the last lane before them, then the upper half lane 31
}
template <typename Units>
__device__ __forceinline__ KvItem kv_item(const KvBatch &t, int item, Units units) {      // units(count, value): items of a sequence
    const int lane = threadIdx.x & 63;
    KvItem got{0, -1, 0, 0, 0};
    for (int b0 = 0; b0 < t.sequences; b0 += 64) {
        const int b = b0 + lane < t.sequences ? b0 + lane : t.sequences - 1;
        const int first = kv_within(t.cu[b], 0, t.total), count = kv_within(t.cu[b + 1], first, t.total) - first, value = t.kv_len[b];
        const int mine = b0 + lane < t.sequences ? units(count, value) : 0;
        const int upto = kv_sum_upto(mine);
        const unsigned long long past = __builtin_amdgcn_ballot_w64(upto > item);
        if (past != 0ull) {
            const int at = __builtin_ctzll(past);
            got.sequence = b0 + at;
            const int local = item - __builtin_amdgcn_readlane(upto - mine, at);
            got.local = (uint32_t)local < (uint32_t)__builtin_amdgcn_readlane(mine, at) ? local : -1;      // (counts that do not ascend may sum past 32 bits)
            got.first = __builtin_amdgcn_readlane(first, at);
            got.count = __builtin_amdgcn_readlane(count, at);
            got.value = __builtin_amdgcn_readlane(value, at);
            break;
        }
        item -= __builtin_amdgcn_readlane(upto, 63);
    }
    return got;
}
// sequence b's tokens within 0 .. total
__device__ __forceinline__ void kv_range(const int32_t *cu, int b, int total, int &first, int &count) {
    const int lo = kv_within(cu[b], 0, total), hi = kv_within(cu[b + 1], lo, total);
    first = __builtin_amdgcn_readfirstlane(lo);
    count = __builtin_amdgcn_readfirstlane(hi - lo);
}
// tokens of a sequence that the cache can hold
__device__ __forceinline__ int kv_length(const KvCache &c, const KvBatch &t, int len) {
    const long long most = (long long)t.table_width << c.page_shift;
    return len < 0 ? 0 : (long long)len > most ? (int)most : len;
}
// (page, head, block within the page) of block `blk` of sequence b as an index of the scale arrays, -1 where the table names no page of the cache
__device__ __forceinline__ long long kv_unit(const KvCache &c, const int32_t *table, int width, int b, int head, int blk) {
    const int bs = c.page_shift - 5;
    const int page = table[(size_t)b * width + (blk >> bs)];
    if ((uint32_t)page >= (uint32_t)c.pages) return -1;
    return (((long long)page * c.heads + head) << bs) + (blk & ((1 << bs) - 1));
}

// ---- E4M3 -------------------------------------------------------------------------------------------------------------------
__device__ __forceinline__ float kv_pow2(int e) {      // 2^e, 0 below the smallest normal number
    return e < -126 ? 0.f : __uint_as_float((uint32_t)(e + 127) << 23);
}
// the byte of the smallest power of two s >= 2^-126 with amax <= 448 s = 1.75 * 2^8 s, from the bits of a finite maximum
__device__ __forceinline__ int kv_scale_byte(uint32_t amax_bits) {
    const int byte = (int)(amax_bits >> 23) - 8 + ((amax_bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    return amax_bits == 0u ? 0 : byte < 1 ? 1 : byte;
}
// four numbers of at most 448 in magnitude as four codes, round to nearest even
__device__ __forceinline__ uint32_t kv_codes4(float a, float b, float c, float d) {
    int w = 0;
    w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, w, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
// four codes of a block whose scale grew by 2^-e
__device__ __forceinline__ uint32_t kv_rescale4(uint32_t w, float factor) {
    const kv_floatx2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    return kv_codes4(lo[0] * factor, lo[1] * factor, hi[0] * factor, hi[1] * factor);
}
// eight codes times a power of two as f16 (exact within its range)
__device__ __forceinline__ kv_f16x8 kv_f16_of(uint32_t lo, uint32_t hi, float scale) {
    const kv_f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, scale, true);
    const kv_f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, scale, true);
    return kv_f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// ---- rotation ---------------------------------------------------------------------------------------------------------------
__device__ __forceinline__ void kv_floats(uint4 w, float (&x)[8]) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(u[i] << 16);
        x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void kv_load8(const float *p, float (&x)[8]) {
    const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
// Two channels of a pair: (a, b) -> (a c - b s, b c + a s), each product and the sum rounded once (the build contracts nothing).
__device__ __forceinline__ float kv_turn_a(float a, float b, float c, float s) { return a * c - b * s; }
__device__ __forceinline__ float kv_turn_b(float a, float b, float c, float s) { return b * c + a * s; }

// Eight channels at each of N places of one row of 16-bit queries at position `pos`, rotated, in fp32; place(i) is a multiple of 8.  In the order of halves
// the partners of eight neighbours are eight neighbours, in the interleaved order they are among themselves (dims is a multiple of 16).  Everything
// is requested before the first is used; channels past `dims` are loaded like the others and left as they are.
template <int N>
struct KvRotating {
    uint4 own[N], other[N];
    float c[N][8], s[N][8];
    template <typename Place>
    __device__ __forceinline__ void request(const uint16_t *row, const KvRope &rope, int pos, Place place) {
#pragma unroll
        for (int i = 0; i < N; ++i) own[i] = *reinterpret_cast<const uint4 *>(row + place(i));
        if (rope.dims == 0) return;
        const float *t = rope.table + (size_t)(pos < 0 ? 0 : pos < rope.positions ? pos : rope.positions - 1) * rope.dims;
        const int half = rope.dims / 2;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int d = place(i) < rope.dims ? place(i) : 0;
            const int first = rope.interleaved ? d / 2 : d >= half ? d - half : d;
            other[i] = own[i];
            if (!rope.interleaved) other[i] = *reinterpret_cast<const uint4 *>(row + (d >= half ? d - half : d + half));
            // (interleaved: the first four of each)
            const float4 c0 = *reinterpret_cast<const float4 *>(t + first), s0 = *reinterpret_cast<const float4 *>(t + half + first);
            const int more = rope.interleaved ? 0 : 4;
            const float4 c1 = *reinterpret_cast<const float4 *>(t + first + more), s1 = *reinterpret_cast<const float4 *>(t + half + first + more);
            c[i][0] = c0.x; c[i][1] = c0.y; c[i][2] = c0.z; c[i][3] = c0.w; c[i][4] = c1.x; c[i][5] = c1.y; c[i][6] = c1.z; c[i][7] = c1.w;
            s[i][0] = s0.x; s[i][1] = s0.y; s[i][2] = s0.z; s[i][3] = s0.w; s[i][4] = s1.x; s[i][5] = s1.y; s[i][6] = s1.z; s[i][7] = s1.w;
        }
    }
    template <typename Place>
    __device__ __forceinline__ void finish(const KvRope &rope, Place place, float (&x)[N][8]) const {
#pragma unroll
        for (int i = 0; i < N; ++i) kv_floats(own[i], x[i]);
        if (rope.dims == 0) return;
        if (rope.interleaved) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const bool turn = place(i) < rope.dims;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float a = x[i][2 * e], b = x[i][2 * e + 1];
                    x[i][2 * e] = turn ? kv_turn_a(a, b, c[i][e], s[i][e]) : a;
                    x[i][2 * e + 1] = turn ? kv_turn_b(a, b, c[i][e], s[i][e]) : b;
                }
            }
            return;
        }
        const int half = rope.dims / 2;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float y[8];
            kv_floats(other[i], y);
            const bool turn = place(i) < rope.dims, second = place(i) >= half;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float z = second ? kv_turn_b(y[e], x[i][e], c[i][e], s[i][e]) : kv_turn_a(x[i][e], y[e], c[i][e], s[i][e]);
                x[i][e] = turn ? z : x[i][e];
            }
        }
    }
};
// Barrier of a workgroup for what its wavefronts wrote to LDS: loads from memory stay in flight.
__device__ __forceinline__ void kv_lds_barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// ---- reductions over the lane groups of a wavefront: every lane gets the result (v_permlane32_swap / v_permlane16_swap of a register with itself
// leaves one operand of each pair of halves, or of rows, in both) -------------------------------------------------------------
__device__ __forceinline__ void kv_swap32(float x, float &a, float &b) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    a = __uint_as_float(r[0]);
    b = __uint_as_float(r[1]);
}
__device__ __forceinline__ void kv_swap16(float x, float &a, float &b) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    a = __uint_as_float(r[0]);
    b = __uint_as_float(r[1]);
}
__device__ __forceinline__ float kv_max32(float x) { float a, b; kv_swap32(x, a, b); return fmaxf(a, b); }
__device__ __forceinline__ float kv_max16(float x) { float a, b; kv_swap16(x, a, b); return fmaxf(a, b); }
// over U = 4, 8 or 16 neighbouring lanes, NaN if one is NaN
template <int CONTROL>
__device__ __forceinline__ float kv_max_dpp(float x) {
    const int y = __builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CONTROL, 0xf, 0xf, false);
    return __builtin_elementwise_maximum(x, __uint_as_float((uint32_t)y));
}
template <int U>
__device__ __forceinline__ float kv_max_lanes(float x) {
    x = kv_max_dpp<0x4e>(kv_max_dpp<0xb1>(x));      // quads: lanes 1, 0, 3, 2, then 2, 3, 0, 1
    if (U >= 8) x = kv_max_dpp<0x141>(x);           // eight lanes backwards
    if (U >= 16) x = kv_max_dpp<0x140>(x);          // sixteen
    return x;
}
__device__ __forceinline__ float kv_within_range(float x) { return __builtin_elementwise_maximum(__builtin_elementwise_minimum(x, 3.4028235e38f), -3.4028235e38f); }      // (NaN stays)
// 1 / the sum of a row's weights, within an ulp (no key seen: zeros; NaN stays).  (The division proper is a chain of ten instructions, twice or three times a launch.)
__device__ __forceinline__ float kv_inverse(float sum) { return sum > 0.f ? __builtin_amdgcn_rcpf(sum) : sum == sum ? 0.f : sum; }
__device__ __forceinline__ float kv_sum32(float x) { float a, b; kv_swap32(x, a, b); return a + b; }
__device__ __forceinline__ float kv_sum16(float x) { float a, b; kv_swap16(x, a, b); return a + b; }

// ---- values of very different scales -------------------------------------------------------------------------------------------
// Values go to the matrix cores as f16, code * 2^(byte - reference) with the largest byte as the reference.  A code is a multiple of 2^-9 and f16 has multiples of 2^-24, so
// that is exact while the bytes are at most 15 apart, whichever of the blocks a row sees.  Where they are farther apart (blocks of zeros aside), a kernel takes its other
// way: every block of 32 by itself, its codes as they are, its weights relative to the largest in the block; per row the sums so far and the block's meet in fp32
// with an exponent of their own.  What a row does not see, or gives no weight, then leaves no trace in it.
// It costs 1.2 times the time for few rows and four times for many (8192 tokens on 16384 keys 6.5 ms).
constexpr int kKvExactSpread = 15;
struct KvSpread {
    int lo = 255, hi = 0, first = 0;      // of the lane; a byte that some block has
    __device__ __forceinline__ bool add(int byte) {      // a byte in every lane, 0: none.  Whether all so far are too far apart
        hi = byte > hi ? byte : hi;
        lo = byte != 0 && byte < lo ? byte : lo;
        if (first == 0) {
            const unsigned long long some = __builtin_amdgcn_ballot_w64(byte != 0);
            first = some != 0ull ? __builtin_amdgcn_readlane(byte, __builtin_ctzll(some)) : 0;
        }
        if (__builtin_amdgcn_ballot_w64(hi > first + kKvExactSpread / 2 || lo < first - kKvExactSpread / 2) == 0ull) return false;      // (mostly they are near any of them)
        const float up = kv_max32(kv_max16(kv_max_lanes<16>((float)hi))), down = kv_max32(kv_max16(kv_max_lanes<16>((float)-lo)));
        return __builtin_amdgcn_readfirstlane((int)up) + __builtin_amdgcn_readfirstlane((int)down) > kKvExactSpread;
    }
};
// sums = ldexp(sums * keep, keep_e) + ldexp(block * add, add_e), weights = weights * keep_l + block * add_l
struct KvJoin { float keep, add, keep_l, add_l; int keep_e, add_e; };
// Row by row: m: maximum so far; sums stand for sums * 2^(ref - 127) and reach `largest`; the block has maximum `top` (-inf: the row sees none of it) and byte `byte`.
// Sums are brought near 2^30 or below the block's 2^22, whichever leaves neither past fp32.
__device__ __forceinline__ KvJoin kv_join(float &m, int &ref, float top, int byte, float largest) {
    const bool none = !(top > -__builtin_inff());
    const float m_new = none ? m : fmaxf(m, top), x = none ? 0.f : top - m_new, k = m - m_new;
    const float xi = fmaxf(__builtin_floorf(x), -20000.f), ki = fmaxf(__builtin_floorf(k), -20000.f);
    const int block = byte + (int)xi, sums = ref + (int)ki + __builtin_amdgcn_frexp_expf(largest) - 30;
    const int ref_new = none ? ref : largest > 0.f && sums > block ? sums : block;
    const KvJoin j = {__builtin_amdgcn_exp2f(k - ki), none ? 0.f : __builtin_amdgcn_exp2f(x - xi), __builtin_amdgcn_exp2f(k), none ? 0.f : __builtin_amdgcn_exp2f(x),
                      ref + (int)ki - ref_new, block - ref_new};
    m = m_new;
    ref = ref_new;
    return j;
}

}  // namespace svdq
