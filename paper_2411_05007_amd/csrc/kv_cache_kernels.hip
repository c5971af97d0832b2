// Writing the paged 8-bit cache of keys and values, and reading it back (layout: kv_common.h).
//
// Append.  x' = the rotation of a key by its position (values as they are); per block of 32 tokens and head: byte = that of the smallest power of
// two s with max|x'| <= 448 s, or the block's own if that is larger; code = e4m3(x' / s), round to nearest even.  Division by a power of
// two is exact, so the one rounding of a code is the format's; a block that is filled over several calls keeps its codes while its byte stays and rounds
// them once more when it grows (which changes only codes that become subnormal).  A vector with an element that is not finite does not take part in the maximum
// and is stored as NaN codes in the keys and zeros in the values of its token and head: every query that sees the token gets NaN and no
// other does, though the values of masked tokens are multiplied by zero.
// Work split: a workgroup of four wavefronts has one block of a sequence and one to four heads in turn, two wavefronts the keys and two the values, 16 tokens each: a
// maximum is a reduction within a wavefront and one exchange through LDS, which carries the mask of vectors that are not finite too.  One workgroup owns a block
// of a head; within it a wavefront reads and writes the codes of its own tokens only, and the byte that the block has is read by one wavefront of a side, which tells both through
// LDS and writes the new one behind the barrier of that exchange.  The rows of the next head are in flight while one is worked on.
// Bound: memory (4 bytes read and 2 written per channel of a token) with many tokens, if the instructions stay few: conversions take the scale with them and two
// numbers at a time, magnitudes of values are compared two at a time as integers, places and the rotation's cosines are found once for all heads.
// 4 x 4608 tokens, 24 heads of 128: 83 us, 5.1 TB/s (one head a workgroup 103, three 83, six 83; scaled and converted apart 105).  For few tokens a chain of round
// trips (lengths, block table, codes that are there): 64 tokens, 8 heads of 128 are 7.3 us; 12 heads of 64, 5120 tokens 10.1 us.
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

// The keys of half a block, 16 tokens.  A unit is 16 channels of a token, the two runs of eight that the rotation pairs; a lane has N of them.
// (Per head and wavefront the instructions are what counts: places are found once for all heads, relative to a base that is the same for all lanes.)
template <int D>
struct KeySide {
    static constexpr int U = D / 16, N = U / 4, kRaw = N * 8;
    const KvAppendParams &p;
    const BlockWork &w;
    const int lane, half;
    const uint16_t *base;         // of the block's first new token and head 0
    uint32_t from[N][2], to[N][2];      // places in the rows, from there, and in the codes of a block
    uint32_t raw[kRaw];
    float c[N][8], s[N][8], x[N][2][8];
    float top[N];
    __device__ __forceinline__ int token(int i) const { return 16 * half + (lane + 64 * i) / U; }
    __device__ __forceinline__ KeySide(const KvAppendParams &p_, const BlockWork &w_, int lane_, int half_) : p(p_), w(w_), lane(lane_), half(half_) {
        base = p.k.data + (w.row0 + w.lo) * p.k.token_stride;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int pr = (lane + 64 * i) % U;
            const bool halves = !p.rope.interleaved && pr < p.rope.dims / 16;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int d = halves ? pr * 8 + j * (p.rope.dims / 2) : pr * 16 + j * 8;
                from[i][j] = (uint32_t)(readable(w, token(i)) - w.lo) * (uint32_t)p.k.token_stride + (uint32_t)d;
                to[i][j] = (uint32_t)(token(i) * D + d);
            }
        }
    }
    __device__ __forceinline__ void load_common() {      // the same for all heads
        if (p.rope.dims == 0) return;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int last = p.rope.dims / 16 - 1, pr = (lane + 64 * i) % U, pos = w.blk * kKvBlock + readable(w, token(i));
            const float *t = p.rope.table + (size_t)(pos < p.rope.positions ? pos : p.rope.positions - 1) * p.rope.dims + (pr < last ? pr : last) * 8;
            kv_load8(t, c[i]);
            kv_load8(t + p.rope.dims / 2, s[i]);
        }
    }
    __device__ __forceinline__ void load(uint32_t (&r)[kRaw], int h) const {
        const uint16_t *head = base + h * p.k.head_stride;
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const uint4 v = *reinterpret_cast<const uint4 *>(head + from[i][j]);
                r[i * 8 + j * 4] = v.x; r[i * 8 + j * 4 + 1] = v.y; r[i * 8 + j * 4 + 2] = v.z; r[i * 8 + j * 4 + 3] = v.w;
            }
    }
    __device__ __forceinline__ void load_old(long long) {}
    // turns the rows; returns the tokens with an element that is not finite (top: largest magnitude of a unit)
    __device__ __forceinline__ uint32_t look() {
        uint32_t bad = 0u;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            kv_floats(make_uint4(raw[i * 8], raw[i * 8 + 1], raw[i * 8 + 2], raw[i * 8 + 3]), x[i][0]);
            kv_floats(make_uint4(raw[i * 8 + 4], raw[i * 8 + 5], raw[i * 8 + 6], raw[i * 8 + 7]), x[i][1]);
            if ((lane + 64 * i) % U < p.rope.dims / 16) {
                if (p.rope.interleaved) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float a = x[i][e / 4][2 * (e % 4)], y = x[i][e / 4][2 * (e % 4) + 1];
                        x[i][e / 4][2 * (e % 4)] = kv_turn_a(a, y, c[i][e], s[i][e]);
                        x[i][e / 4][2 * (e % 4) + 1] = kv_turn_b(a, y, c[i][e], s[i][e]);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float a = x[i][0][e], y = x[i][1][e];
                        x[i][0][e] = kv_turn_a(a, y, c[i][e], s[i][e]);
                        x[i][1][e] = kv_turn_b(a, y, c[i][e], s[i][e]);
                    }
                }
            }
            float m = 0.f;      // (NaN if one is NaN)
#pragma unroll
            for (int e = 0; e < 8; ++e) m = __builtin_elementwise_maximum(__builtin_elementwise_maximum(m, __builtin_fabsf(x[i][0][e])), __builtin_fabsf(x[i][1][e]));
            top[i] = live(w, token(i)) ? m : 0.f;
            bad |= abs_bits(top[i]) >= kInfBits ? 1u << token(i) : 0u;
        }
        return any_bits_64(bad);
    }
    __device__ __forceinline__ uint32_t largest(uint32_t bad) const {
        uint32_t m = 0u;
#pragma unroll
        for (int i = 0; i < N; ++i) m = umax(m, (bad >> token(i)) & 1u ? 0u : abs_bits(top[i]));
        return max_bits_64(m);
    }
    __device__ __forceinline__ void write(long long unit, const BlockScale &sc, uint32_t bad) {
        uint8_t *codes = p.cache.k + (size_t)unit * (32 * D);
        if (w.lo > 0 && sc.grown) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (token(i) < w.lo)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        uint2 *dst = reinterpret_cast<uint2 *>(codes + to[i][j]);
                        const uint2 v = *dst;
                        *dst = make_uint2(kv_rescale4(v.x, sc.old_factor), kv_rescale4(v.y, sc.old_factor));
                    }
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            uint2 v[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float (&y)[8] = x[i][j];
                v[j] = make_uint2(codes4(y[0], y[1], y[2], y[3], sc.scale), codes4(y[4], y[5], y[6], y[7], sc.scale));
                if (bad != 0u && (bad >> token(i)) & 1u) v[j].x = v[j].y = kKvNaN * 0x01010101u;
            }
            if (!live(w, token(i))) continue;
            *reinterpret_cast<uint2 *>(codes + to[i][0]) = v[0];
            *reinterpret_cast<uint2 *>(codes + to[i][1]) = v[1];
        }
    }
};

// The values of half a block, two slots.  A lane has the eight tokens of a slot for E channels: what it writes is E runs of eight bytes.
template <int D>
struct ValueSide {
    static constexpr int E = D / 32, Q = 16 / E, W = E / 2, kRaw = 8 * W;
    const KvAppendParams &p;
    const BlockWork &w;
    const int lane, half, slot;
    const uint16_t *base;
    uint32_t from[8], to;
    uint32_t fresh[2], keep[2];      // bytes of a run: new ones, and those that are there
    uint32_t raw[kRaw];
    uint2 old[E];
    __device__ __forceinline__ int token(int j) const { return kv_slot_token(slot) + (j & 3) + 8 * (j >> 2); }
    __device__ __forceinline__ ValueSide(const KvAppendParams &p_, const BlockWork &w_, int lane_, int half_) : p(p_), w(w_), lane(lane_), half(half_), slot(2 * half_ + (lane_ & 1)) {
        const int a = (lane >> 2) / Q, c = (lane >> 1) & 1, q = (lane >> 2) % Q;
        base = p.v.data + (w.row0 + w.lo) * p.v.token_stride;
        to = (uint32_t)(((a * 16 + E * q) * 4 + slot) * 16 + 8 * c);
        fresh[0] = fresh[1] = keep[0] = keep[1] = 0u;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            from[j] = (uint32_t)(readable(w, token(j)) - w.lo) * (uint32_t)p.v.token_stride + (uint32_t)(32 * a + 16 * c + E * q);
            if (live(w, token(j))) fresh[j >> 2] |= 0xffu << (8 * (j & 3));
            if (token(j) < w.lo) keep[j >> 2] |= 0xffu << (8 * (j & 3));
        }
    }
    __device__ __forceinline__ void load_common() {}
    __device__ __forceinline__ void load(uint32_t (&r)[kRaw], int h) const {
        const uint16_t *head = base + h * p.v.head_stride;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const typename RawOf<E>::type v = *reinterpret_cast<const typename RawOf<E>::type *>(head + from[j]);
            __builtin_memcpy(r + j * W, &v, sizeof v);
        }
    }
    __device__ __forceinline__ void load_old(long long unit) {
        if (w.lo == 0) return;
#pragma unroll
        for (int e = 0; e < E; ++e) old[e] = *reinterpret_cast<const uint2 *>(p.cache.v + (size_t)unit * (32 * D) + to + 64 * e);
    }
    // largest magnitude of a token's channels, as bf16 bits
    __device__ __forceinline__ uint32_t largest_of(int j) const {
        uint32_t m = raw[j * W] & 0x7fff7fffu;
#pragma unroll
        for (int i = 1; i < W; ++i) m = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(ushort2_t, m), __builtin_bit_cast(ushort2_t, raw[j * W + i] & 0x7fff7fffu)));
        return live(w, token(j)) ? m : 0u;
    }
    __device__ __forceinline__ uint32_t look() {
        uint32_t m = 0u;
#pragma unroll
        for (int j = 0; j < 8; ++j) m = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(ushort2_t, m), __builtin_bit_cast(ushort2_t, largest_of(j))));
        if (__builtin_amdgcn_ballot_w64((m << 16) >= kInfBits || m >= kInfBits) == 0ull) return 0u;
        uint32_t bad = 0u;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t t = largest_of(j);
            bad |= (t << 16) >= kInfBits || t >= kInfBits ? 1u << token(j) : 0u;
        }
        return any_bits_64(bad);
    }
    __device__ __forceinline__ uint32_t largest(uint32_t bad) const {
        uint32_t m = 0u;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            m = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(ushort2_t, m), __builtin_bit_cast(ushort2_t, bad != 0u && (bad >> token(j)) & 1u ? 0u : largest_of(j))));
        return max_bits_64(umax(m << 16, m & 0xffff0000u));
    }
    __device__ __forceinline__ void write(long long unit, const BlockScale &sc, uint32_t bad) {
        uint32_t mask[2] = {fresh[0], fresh[1]};      // (a vector that is not finite is cleared; its conversion may overflow)
        if (bad != 0u) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if ((bad >> token(j)) & 1u) mask[j >> 2] &= ~(0xffu << (8 * (j & 3)));
        }
        if (w.lo > 0 && sc.grown) {
#pragma unroll
            for (int e = 0; e < E; ++e) old[e] = make_uint2(kv_rescale4(old[e].x, sc.old_factor), kv_rescale4(old[e].y, sc.old_factor));
        }
        uint8_t *codes = p.cache.v + (size_t)unit * (32 * D) + to;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const uint32_t pick = e % 2 ? 0x07060302u : 0x05040100u;      // the channel's bf16 numbers of two tokens
            uint32_t v[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t *r = raw + 4 * i * W + e / 2;
                v[i] = codes4(__builtin_amdgcn_perm(r[W], r[0], pick), __builtin_amdgcn_perm(r[3 * W], r[2 * W], pick), sc.scale) & mask[i];
                if (w.lo > 0) v[i] |= (i ? old[e].y : old[e].x) & keep[i];
            }
            *reinterpret_cast<uint2 *>(codes + 64 * e) = make_uint2(v[0], v[1]);
        }
    }
};

// Rows first, then what waits for the block table; the rows of the next head are requested before this one's are worked on.  The four wavefronts' masks and
// maxima meet once a head.
template <typename Side>
__device__ __forceinline__ void append_heads(const KvAppendParams &p, const BlockWork &w, int sequence, int h0, int h1, uint8_t *scales, int wave, Exchange (&exchange)[2]) {
    Side side(p, w, (int)threadIdx.x & 63, wave & 1);
    side.load(side.raw, h0);
    side.load_common();
    const long long unit0 = kv_unit(p.cache, p.batch.table, p.batch.table_width, sequence, h0, w.blk);
    if (unit0 < 0) return;     // (all wavefronts)
    for (int h = h0; h < h1; ++h) {
        uint32_t next[Side::kRaw];
        side.load(next, h + 1 < h1 ? h + 1 : h);
        const long long unit = unit0 + ((long long)(h - h0) << (p.cache.page_shift - 5));
        const bool tells = side.lane == 0 && (wave & 1) == 0;      // of the side's byte, old and new
        const int held = tells && w.lo > 0 ? (int)scales[unit] : 0;
        side.load_old(unit);
        Exchange &ex = exchange[h & 1];      // (written again two heads on: behind a barrier that every wavefront enters when it has read it)
        const uint32_t bad = side.look(), most = side.largest(bad);
        if (side.lane == 0) {
            ex.bad[wave] = bad;
            ex.top[wave] = most;
        }
        if (tells) ex.old_byte[wave >> 1] = held;
        kv_lds_barrier();
        const uint32_t all = ex.bad[0] | ex.bad[1] | ex.bad[2] | ex.bad[3];
        if (all != 0u) {           // (what the other side found is left out of this side's maximum too)
            kv_lds_barrier();      // the words above are read
            const uint32_t again = side.largest(all);
            if (side.lane == 0) ex.top[wave] = again;
            kv_lds_barrier();
        }
        const BlockScale sc = block_scale(umax(ex.top[wave & 2], ex.top[(wave & 2) + 1]), __builtin_amdgcn_readfirstlane(ex.old_byte[wave >> 1]));
        side.write(unit, sc, all);
        if (tells) scales[unit] = (uint8_t)sc.byte;
#pragma unroll
        for (int i = 0; i < Side::kRaw; ++i) side.raw[i] = next[i];
    }
}

template <int D>
__global__ __launch_bounds__(256) void kv_append_kernel(KvAppendParams p, int heads_per_wg) {
    __shared__ Exchange exchange[2];
    const KvItem item = kv_item(p.batch, blockIdx.x, [&](int n, int value) {
        const int len = kv_length(p.cache, p.batch, value), first = len > n ? len - n : 0;
        return n > 0 ? ((len + 31) >> 5) - (first >> 5) : 0;
    });
    const int n = item.count, len = kv_length(p.cache, p.batch, item.value), before = len - n;      // (before < 0: the first -before tokens have no place in the sequence)
    const int first_pos = before < 0 ? 0 : before;
    BlockWork w;
    w.blk = (first_pos >> 5) + item.local;
    if (item.local < 0 || w.blk * kKvBlock >= len || n == 0) return;
    w.lo = first_pos > w.blk * kKvBlock ? first_pos - w.blk * kKvBlock : 0;
    w.hi = len - w.blk * kKvBlock < kKvBlock ? len - w.blk * kKvBlock : kKvBlock;
    w.row0 = (long long)item.first + (w.blk * kKvBlock - before);      // input row of the block's token 0 (rows lo .. hi - 1 are read)
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h0 = blockIdx.y * heads_per_wg, h1 = h0 + heads_per_wg < p.cache.heads ? h0 + heads_per_wg : p.cache.heads;
    if (wave < 2) append_heads<KeySide<D>>(p, w, item.sequence, h0, h1, p.cache.ks, wave, exchange);
    else append_heads<ValueSide<D>>(p, w, item.sequence, h0, h1, p.cache.vs, wave, exchange);
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
    // (past 2^30 no table names a page: places of tokens stay within 32 bits)
    const auto start_of = [](int value) { return kv_within(value, 0, 1 << 30); };
    const KvItem item = kv_item(p.batch, blockIdx.x, [&](int n, int value) {
        const long long start = start_of(value);
        return n > 0 ? (int)((start + n + 31) / 32 - start / 32) : 0;
    });
    const int b = item.sequence, local = item.local, r0 = item.first, n = item.count, start = start_of(item.value);
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
    // Heads a workgroup: one while there are fewer workgroups than stay on the chip together (256 CUs, four each), then more, up to four, which saves what is the
    // same for all heads.  1, 2, 4 heads: 64 items of 8 heads of 128 7.4, 7.5, 9.5 us; 190 of 12 of 64 11.2, 10.1, 11.5 us; 580 of 24 of 128 103, 88, 83 us.
    const long long rounds = (long long)items * p.cache.heads / 1024;
    const int most = rounds < 1 ? 1 : rounds > 4 ? 4 : (int)rounds, per = most < p.cache.heads ? most : p.cache.heads;
    const dim3 grid(items, (p.cache.heads + per - 1) / per);
    switch (p.cache.dim) {
        case 64: kv_append_kernel<64><<<grid, 256, 0, stream>>>(p, per); break;
        case 128: kv_append_kernel<128><<<grid, 256, 0, stream>>>(p, per); break;
        case 256: kv_append_kernel<256><<<grid, 256, 0, stream>>>(p, per); break;
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
