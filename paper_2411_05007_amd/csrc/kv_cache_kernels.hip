// Writing the paged 8-bit cache of keys and values, and reading it back (layout: kv_common.h).
//
// Append.  x' = the rotation of a key by its position (values as they are); per block of 32 tokens and head: byte = that of the smallest power of
// two s with max|x'| <= 448 s, or the block's own if that is larger; code = e4m3(x' / s), round to nearest even.  Division by a power of
// two is exact, so the one rounding of a code is the format's; a block that is filled over several calls keeps its codes while its byte stays and rounds
// them once more when it grows (which changes only codes that become subnormal).  A vector with an element that is not finite does not take part in the maximum
// and is stored as NaN codes in the keys and zeros in the values of its token and head: every query that sees the token gets NaN and no
// other does, though the values of masked tokens are multiplied by zero.
// Work split: a workgroup of two wavefronts has one block of a sequence for a few heads, wavefront 0 the keys, wavefront 1 the values: the
// maximum is a reduction within a wavefront, and the one exchange between the two is the mask of vectors that are not finite.
// One workgroup owns a block, so there is nothing to race with.  Bound: memory (4 bytes read and 2 written per channel of a token).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.h"
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
__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }
__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }
constexpr uint32_t kInfBits = 0x7f800000u;

template <int N> struct RawOf;      // N 16-bit numbers as they are loaded
template <> struct RawOf<2> { typedef uint32_t type; };
template <> struct RawOf<4> { typedef uint2 type; };
template <> struct RawOf<8> { typedef uint4 type; };
template <int N>
__device__ __forceinline__ void bf16_load(const uint16_t *p, float (&x)[N]) {
    typename RawOf<N>::type w = *reinterpret_cast<const typename RawOf<N>::type *>(p);
    uint32_t u[N / 2];
    __builtin_memcpy(u, &w, sizeof w);
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        x[2 * i] = __uint_as_float(u[i] << 16);
        x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
}

// The block's scale: its byte, and what codes that are in it already are multiplied by (1 if they stay).
struct BlockScale { int byte; float to_code, old_factor; bool grown; };
__device__ __forceinline__ BlockScale block_scale(uint32_t amax_bits, int old_byte) {
    BlockScale s;
    const int b = kv_scale_byte(amax_bits);
    s.byte = b > old_byte ? b : old_byte;
    s.grown = s.byte > old_byte;
    s.to_code = kv_pow2(127 - (s.byte < 1 ? 1 : s.byte));
    s.old_factor = kv_pow2(old_byte - s.byte < -100 ? -100 : old_byte - s.byte);
    return s;
}

template <int D>
__global__ __launch_bounds__(128) void kv_append_kernel(KvAppendParams p, int heads_per_wg) {
    __shared__ uint32_t bad_of[2][2];      // vectors that are not finite: [head's parity][keys, values]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const KvItem item = kv_item(p.batch, blockIdx.x, [&](int n, int value) {
        const int len = kv_length(p.cache, p.batch, value), first = len > n ? len - n : 0;
        return n > 0 ? ((len + 31) >> 5) - (first >> 5) : 0;
    });
    const int b = item.sequence, local = item.local, t0 = item.first, n = item.count;
    const int len = kv_length(p.cache, p.batch, item.value), before = len - n;      // (before < 0: the first -before tokens have no place in the sequence)
    const int first_pos = before < 0 ? 0 : before;
    const int blk = (first_pos >> 5) + local;
    if (local < 0 || blk * kKvBlock >= len || n == 0) return;
    // tokens lo .. hi - 1 of the block are new, 0 .. lo - 1 are there already
    const int lo = first_pos > blk * kKvBlock ? first_pos - blk * kKvBlock : 0, hi = len - blk * kKvBlock < kKvBlock ? len - blk * kKvBlock : kKvBlock;
    const long long row0 = (long long)t0 + (blk * kKvBlock - before);       // input row of the block's token 0 (rows lo .. hi - 1 are read)
    const int h0 = blockIdx.y * heads_per_wg, h1 = h0 + heads_per_wg < p.cache.heads ? h0 + heads_per_wg : p.cache.heads;

    for (int h = h0; h < h1; ++h) {
        const long long unit = kv_unit(p.cache, p.batch.table, p.batch.table_width, b, h, blk);
        if (unit < 0) return;      // (the page of a block is the same for all heads)
        if (lane == 0) bad_of[h & 1][wave] = 0u;
        __syncthreads();
        const int old_byte = lo > 0 ? (int)(wave == 0 ? p.cache.ks : p.cache.vs)[unit] : 0;
        if (wave == 0) {
            // unit u of the block: 16 channels of a token, two runs of eight that the rotation pairs
            constexpr int U = D / 16, N = 32 * U / 64;
            float x[N][2][8];
            uint32_t top[N];
            int at[N][2];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int u = lane + 64 * i, tok = u / U, pr = u % U;
                const bool live = tok >= lo && tok < hi;
                const int half = p.rope.dims / 2;
                const bool halves = !p.rope.interleaved && pr < p.rope.dims / 16;
                at[i][0] = halves ? pr * 8 : pr * 16;
                at[i][1] = halves ? pr * 8 + half : pr * 16 + 8;
                top[i] = 0u;
                if (!live) continue;
                const uint16_t *row = p.k.data + (row0 + tok) * p.k.token_stride + h * p.k.head_stride;
                kv_floats(*reinterpret_cast<const uint4 *>(row + at[i][0]), x[i][0]);
                kv_floats(*reinterpret_cast<const uint4 *>(row + at[i][1]), x[i][1]);
                if (at[i][0] < p.rope.dims) {
                    const int pos = blk * kKvBlock + tok;
                    const float *t = p.rope.table + (size_t)(pos < p.rope.positions ? pos : p.rope.positions - 1) * p.rope.dims;
                    float c[8], s[8];
                    kv_load8(t + pr * 8, c);
                    kv_load8(t + half + pr * 8, s);
                    if (halves) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float a = x[i][0][e], y = x[i][1][e];
                            x[i][0][e] = kv_turn_a(a, y, c[e], s[e]);
                            x[i][1][e] = kv_turn_b(a, y, c[e], s[e]);
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            float &a = x[i][e / 4][2 * (e % 4)], &y = x[i][e / 4][2 * (e % 4) + 1];
                            const float a0 = a, y0 = y;
                            a = kv_turn_a(a0, y0, c[e], s[e]);
                            y = kv_turn_b(a0, y0, c[e], s[e]);
                        }
                    }
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) top[i] = umax(top[i], umax(abs_bits(x[i][0][e]), abs_bits(x[i][1][e])));
                if (top[i] >= kInfBits) atomicOr(&bad_of[h & 1][0], 1u << tok);
            }
            __syncthreads();
            const uint32_t bad = bad_of[h & 1][0] | bad_of[h & 1][1];
            uint32_t m = 0u;
#pragma unroll
            for (int i = 0; i < N; ++i) m = umax(m, (bad >> ((lane + 64 * i) / U)) & 1u ? 0u : top[i]);
            const BlockScale s = block_scale(max_bits_64(m), old_byte);
            uint8_t *codes = p.cache.k + (size_t)unit * (32 * D);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int tok = (lane + 64 * i) / U;
                if (tok >= hi) continue;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    uint2 *dst = reinterpret_cast<uint2 *>(codes + tok * D + at[i][j]);
                    uint2 w;
                    if (tok >= lo) {
                        const float (&y)[8] = x[i][j];
                        w.x = kv_codes4(y[0] * s.to_code, y[1] * s.to_code, y[2] * s.to_code, y[3] * s.to_code);
                        w.y = kv_codes4(y[4] * s.to_code, y[5] * s.to_code, y[6] * s.to_code, y[7] * s.to_code);
                        if ((bad >> tok) & 1u) w.x = w.y = kKvNaN * 0x01010101u;
                        *dst = w;
                    } else if (s.grown) {
                        w = *dst;
                        w.x = kv_rescale4(w.x, s.old_factor);
                        w.y = kv_rescale4(w.y, s.old_factor);
                        *dst = w;
                    }
                }
            }
            if (lane == 0) p.cache.ks[unit] = (uint8_t)s.byte;
        } else {
            // a lane has the eight tokens of one slot for E channels and the E channels sixteen further on: what it writes is E runs of 16 bytes
            constexpr int E = D / 32, Q = 16 / E;
            const int g = lane & 3, a = (lane >> 2) / Q, q = (lane >> 2) % Q, d0 = 32 * a + E * q;
            float x[8][2][E];
            uint32_t top[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int tok = kv_slot_token(g) + (j & 3) + 8 * (j >> 2);
                top[j] = 0u;
                if (tok < lo || tok >= hi) {
#pragma unroll
                    for (int e = 0; e < E; ++e) x[j][0][e] = x[j][1][e] = 0.f;
                    continue;
                }
                const uint16_t *row = p.v.data + (row0 + tok) * p.v.token_stride + h * p.v.head_stride;
                bf16_load<E>(row + d0, x[j][0]);
                bf16_load<E>(row + d0 + 16, x[j][1]);
#pragma unroll
                for (int e = 0; e < E; ++e) top[j] = umax(top[j], umax(abs_bits(x[j][0][e]), abs_bits(x[j][1][e])));
                if (top[j] >= kInfBits) atomicOr(&bad_of[h & 1][1], 1u << tok);
            }
            __syncthreads();
            const uint32_t bad = bad_of[h & 1][0] | bad_of[h & 1][1];
            uint32_t m = 0u;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (!((bad >> (kv_slot_token(g) + (j & 3) + 8 * (j >> 2))) & 1u)) m = umax(m, top[j]);
            const BlockScale s = block_scale(max_bits_64(m), old_byte);
            uint8_t *codes = p.cache.v + (size_t)unit * (32 * D);
            // bytes of the runs that hold new tokens; codes of bad ones are zero
            uint32_t fresh[2], keep[2];
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                fresh[w] = keep[w] = 0u;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int tok = kv_slot_token(g) + k + 8 * w;
                    if (tok >= lo && tok < hi && !((bad >> tok) & 1u)) fresh[w] |= 0xffu << (8 * k);
                    if (tok < lo) keep[w] |= 0xffu << (8 * k);
                }
            }
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int d16 = E * q + e;
                uint4 *dst = reinterpret_cast<uint4 *>(codes + ((a * 16 + d16) * 4 + g) * 16);
                uint32_t w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int c = i / 2, j = 4 * (i % 2);
                    // (a vector that is not finite is cleared below; its conversion may overflow)
                    w[i] = kv_codes4(x[j][c][e] * s.to_code, x[j + 1][c][e] * s.to_code, x[j + 2][c][e] * s.to_code, x[j + 3][c][e] * s.to_code) & fresh[i % 2];
                }
                if (lo > 0) {
                    const uint4 old = *dst;
                    uint32_t o[4] = {old.x, old.y, old.z, old.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[i] |= (s.grown ? kv_rescale4(o[i], s.old_factor) : o[i]) & keep[i % 2];
                }
                *dst = make_uint4(w[0], w[1], w[2], w[3]);
            }
            if (lane == 0) p.cache.vs[unit] = (uint8_t)s.byte;
        }
    }
}

// Gather: rows of the cache as bf16, code * 2^(byte - 127), exact where the product is a normal bf16.  Wavefront 0 has a block's keys, wavefront 1 its values:
// a lane takes eight channels of the eight tokens of a slot, pairs the codes of neighbouring channels with byte permutes, and
// converts two at a time.  Bound: memory (2 bytes read and 4 written per channel of a token).
__device__ __forceinline__ uint32_t bf16_pair(uint32_t w, float scale, bool high) {
    const kv_bf16x2 r = high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false);
    return __builtin_bit_cast(uint32_t, r);
}

template <int D>
__global__ __launch_bounds__(128) void kv_gather_kernel(KvGatherParams p) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const KvItem item = kv_item(p.batch, blockIdx.x, [](int n, int value) {
        const long long start = value < 0 ? 0 : value;
        return n > 0 ? (int)((start + n + 31) / 32 - start / 32) : 0;
    });
    const int b = item.sequence, local = item.local, r0 = item.first, n = item.count, start = item.value < 0 ? 0 : item.value;
    const int blk = (start >> 5) + local;
    const long long end = (long long)start + n;
    if (local < 0 || n == 0 || (long long)blk * kKvBlock >= end) return;
    const int h = blockIdx.y;
    const int lo = start > blk * kKvBlock ? start - blk * kKvBlock : 0, hi = end - (long long)blk * kKvBlock < kKvBlock ? (int)(end - (long long)blk * kKvBlock) : kKvBlock;
    const long long unit = (blk >> (p.cache.page_shift - 5)) < p.batch.table_width ? kv_unit(p.cache, p.batch.table, p.batch.table_width, b, h, blk) : -1;
    uint16_t *out = wave == 0 ? p.k : p.v;
    if (!out) return;
    out += ((size_t)r0 + (size_t)(blk * kKvBlock - start)) * p.cache.heads * D + (size_t)h * D;      // row of the block's token 0 (rows lo .. hi - 1 are written)
    const size_t stride = (size_t)p.cache.heads * D;
    if (unit < 0) {      // no such page: zeros
        for (int i = lane; i < (hi - lo) * (D / 8); i += 64) *reinterpret_cast<uint4 *>(out + (lo + i / (D / 8)) * stride + i % (D / 8) * 8) = make_uint4(0u, 0u, 0u, 0u);
        return;
    }
    const float scale = kv_pow2((int)(wave == 0 ? p.cache.ks : p.cache.vs)[unit] - 127);
    if (wave == 0) {
        const uint8_t *codes = p.cache.k + (size_t)unit * (32 * D);
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {      // 16 channels of a token
            const int u = lane + 64 * i, tok = u / (D / 16), d = u % (D / 16) * 16;
            if (tok < lo || tok >= hi) continue;
            const uint4 w = *reinterpret_cast<const uint4 *>(codes + tok * D + d);
            uint4 *dst = reinterpret_cast<uint4 *>(out + tok * stride + d);
            dst[0] = make_uint4(bf16_pair(w.x, scale, false), bf16_pair(w.x, scale, true), bf16_pair(w.y, scale, false), bf16_pair(w.y, scale, true));
            dst[1] = make_uint4(bf16_pair(w.z, scale, false), bf16_pair(w.z, scale, true), bf16_pair(w.w, scale, false), bf16_pair(w.w, scale, true));
        }
        return;
    }
    const uint8_t *codes = p.cache.v + (size_t)unit * (32 * D);
#pragma unroll
    for (int i = 0; i < (D + 127) / 128; ++i) {
        const int u = lane + 64 * i, g = u / (D / 8), d = u % (D / 8) * 8;      // (D = 64: 32 units)
        if (g >= 4) continue;
        uint2 w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = *reinterpret_cast<const uint2 *>(codes + (((d / 32 * 16 + d % 16 + e) * 4 + g) * 2 + d % 32 / 16) * 8);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            uint32_t row[4][4];      // [token][pair of channels]
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t x = t ? w[2 * e].y : w[2 * e].x, y = t ? w[2 * e + 1].y : w[2 * e + 1].x;
                const uint32_t lo2 = __builtin_amdgcn_perm(y, x, 0x05010400u), hi2 = __builtin_amdgcn_perm(y, x, 0x07030602u);      // tokens 0, 1 and 2, 3
                row[0][e] = bf16_pair(lo2, scale, false);
                row[1][e] = bf16_pair(lo2, scale, true);
                row[2][e] = bf16_pair(hi2, scale, false);
                row[3][e] = bf16_pair(hi2, scale, true);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int tok = kv_slot_token(g) + k + 8 * t;
                if (tok >= lo && tok < hi) *reinterpret_cast<uint4 *>(out + tok * stride + d) = make_uint4(row[k][0], row[k][1], row[k][2], row[k][3]);
            }
        }
    }
}

}  // namespace

hipError_t launch_kv_append(const KvAppendParams &p, hipStream_t stream) {
    const int items = p.batch.total / kKvBlock + 2 * p.batch.sequences;
    int per = 1;
    while (per < 4 && (long long)items * ((p.cache.heads + per - 1) / per) > 4096) per *= 2;
    const dim3 grid(items, (p.cache.heads + per - 1) / per);
    switch (p.cache.dim) {
        case 64: kv_append_kernel<64><<<grid, 128, 0, stream>>>(p, per); break;
        case 128: kv_append_kernel<128><<<grid, 128, 0, stream>>>(p, per); break;
        case 256: kv_append_kernel<256><<<grid, 128, 0, stream>>>(p, per); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

hipError_t launch_kv_gather(const KvGatherParams &p, hipStream_t stream) {
    const dim3 grid(p.batch.total / kKvBlock + 2 * p.batch.sequences, p.cache.heads);
    switch (p.cache.dim) {
        case 64: kv_gather_kernel<64><<<grid, 128, 0, stream>>>(p); break;
        case 128: kv_gather_kernel<128><<<grid, 128, 0, stream>>>(p); break;
        case 256: kv_gather_kernel<256><<<grid, 128, 0, stream>>>(p); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

}  // namespace svdq
