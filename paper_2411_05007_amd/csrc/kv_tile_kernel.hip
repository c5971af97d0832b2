// Attention of many query rows over the paged 8-bit cache: chunks of prompts, joint attention of all tokens of an image (layout: kv_common.h).
//
//   O_i = sum_j softmax_j(scale q'_i . k_j) v_j,   q' the rotated query, j over the keys that row i sees.
//
// The rows of a sequence and key head are its new tokens times the query heads that share the head, so a tile of keys serves the whole group.  A
// workgroup of four wavefronts has 128 rows, 32 to a wavefront; keys and values go by in tiles of 64 tokens, read once per workgroup as codes,
// converted to f16 on the way into LDS (exact: codes of the keys, code * 2^(byte - reference) of the values, the reference exponent the largest seen)
// and laid out as operands, so that an operand read is 64 lanes x 16 bytes in a row.  S^T = K Q^T by v_mfma_f32_32x32x16_f16: a lane has one row of
// queries, its accumulators are the operand of O^T = V^T P^T as they stand, and maximum and sum of a row are one exchange between lane
// halves away.  Statistics in fp32; P is exp2(t - m + 8) in f16, at most 2^14 before the maximum is renewed, so weights down to 2^-22 of the
// largest keep eleven bits; Q in f16, scaled by a power of two per row.
// Bound: the exponentials and the matrix products take turns (per 64 tokens and wavefront 32 matrix instructions and about 250 vector ones).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.h"
#include "kv_common.h"
#include "layout.h"

namespace svdq {
namespace {

constexpr float kNone = -1e30f;
constexpr float kShift = 8.f, kSlack = 6.f;
constexpr int kTileRows = kKvTileRows, kTileKeys = 64;

template <int D>
__global__ __launch_bounds__(256, D > 128 ? 1 : 2) void kv_tile_kernel(KvAttentionParams p) {
    constexpr int C = D / 16, A = D / 32;
    constexpr int N = kTileKeys * D / (256 * 16);      // 16-byte pieces of a tile of codes per thread: 1, 2, 4
    __shared__ __attribute__((aligned(16))) unsigned char kt[kTileKeys * D * 2], vt[kTileKeys * D * 2];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l32 = lane & 31, h32 = lane >> 5;
    const int head = blockIdx.x % p.cache.heads;
    int local, t0, n;
    const int b = kv_item_sequence<1, kTileRows>(p.batch.cu, p.batch.sequences, p.batch.total, p.group, blockIdx.x / p.cache.heads, local);
    kv_range(p.batch.cu, b, p.batch.total, t0, n);
    const int len = kv_length(p.cache, p.batch, b), rows = n * p.group, tiles = (rows + kTileRows - 1) / kTileRows;
    local = __builtin_amdgcn_readfirstlane(local);
    if (local < 0 || local >= tiles) return;
    const int row0 = (p.causal ? tiles - 1 - local : local) * kTileRows;      // (causal: the rows with the most keys first)
    const int r = row0 + wave * 32 + l32 < rows ? row0 + wave * 32 + l32 : rows - 1;
    const int tok = r / p.group, qh = head * p.group + r % p.group, pos = len - n + tok;
    const int seen_hi = p.causal ? (pos + 1 < 0 ? 0 : pos + 1) : len;
    const int seen_lo = p.causal && p.window > 0 && pos + 1 > p.window ? pos + 1 - p.window : 0;
    // keys that some row of the tile, or of the wavefront, sees, and those that all rows of the wavefront see
    auto pos_of = [&](int row) { return len - n + (row < rows ? row : rows - 1) / p.group; };
    auto hi_of = [&](int at) { return p.causal ? (at + 1 < 0 ? 0 : at + 1) : len; };
    auto lo_of = [&](int at) { return p.causal && p.window > 0 && at + 1 > p.window ? at + 1 - p.window : 0; };
    const int wg_lo = lo_of(pos_of(row0)), wg_hi = hi_of(pos_of(row0 + kTileRows - 1));
    const int w_first = pos_of(row0 + wave * 32), w_last = pos_of(row0 + wave * 32 + 31);
    const int any_lo = lo_of(w_first), any_hi = hi_of(w_last), all_lo = lo_of(w_last), all_hi = hi_of(w_first);
    const int key0 = wg_lo / kTileKeys * kTileKeys;

    const int32_t *table = p.batch.table + (size_t)b * p.batch.table_width;
    const int bs = p.cache.page_shift - 5;
    // a tile's two blocks: index of the scale arrays, -1 past the keys or where the table names no page
    auto unit_of = [&](int key) {
        if (key >= wg_hi) return -1ll;
        const int blk = key >> 5, page = table[blk >> bs];
        return (uint32_t)page < (uint32_t)p.cache.pages ? (((long long)page * p.cache.heads + head) << bs) + (blk & ((1 << bs) - 1)) : -1ll;
    };
    struct Tile { uint4 k[N], v[N]; long long unit[2]; int kb[2], vb[2]; };
    auto load = [&](int key) {
        Tile t;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            t.unit[i] = unit_of(key + 32 * i);
            const size_t u = t.unit[i] < 0 ? 0 : (size_t)t.unit[i];
            t.kb[i] = p.cache.ks[u];
            t.vb[i] = p.cache.vs[u];
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int at = (threadIdx.x + 256 * i) * 16, blk = at / (32 * D), in = at % (32 * D);
            const long long at_unit = blk ? t.unit[1] : t.unit[0];
            const size_t u = at_unit < 0 ? 0 : (size_t)at_unit;
            t.k[i] = *reinterpret_cast<const uint4 *>(p.cache.k + u * (32 * D) + in);
            t.v[i] = *reinterpret_cast<const uint4 *>(p.cache.v + u * (32 * D) + in);
        }
        return t;
    };

    kv_f16x8 qf[C];
    float to_t;
    {
        const uint16_t *row = p.q.data + (size_t)(t0 + tok) * p.q.token_stride + qh * p.q.head_stride;
        float x[C][8];
        uint32_t top = 0u;
#pragma unroll
        for (int c = 0; c < C; c += 4) {      // step c: channels 16 c + 8 h32 .. + 7
            kv_rotated<4>(row, p.rope, pos, [&](int i) { return 16 * (c + i) + 8 * h32; }, *reinterpret_cast<float(*)[4][8]>(&x[c]));
            if (c + 4 < C) __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int c = 0; c < C; ++c) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t u = __float_as_uint(x[c][e]) & 0x7fffffffu;
                top = top > u ? top : u;
            }
        }
        const float m = kv_max32(__uint_as_float(top >= 0x7f800000u ? 0x7f800000u : top));
        const int e = (int)(__float_as_uint(m) >> 23) - 127;                          // m in [2^e, 2^(e + 1))
        const int up = e < -100 ? 114 : e > 127 ? 0 : 14 - e;                         // (not finite: as it is, the row becomes NaN)
        const float f = kv_pow2(up);
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) qf[c][i] = (_Float16)(x[c][i] * f);
        to_t = p.scale * kv_pow2(-up);
    }

    kv_floatx16 o[A] = {};
    float m = kNone, l = 0.f;
    int ref = 0;
    Tile cur;
    if (key0 < wg_hi) cur = load(key0);
    for (int key = key0; key < wg_hi; key += kTileKeys) {
        // codes to operands in LDS.  Keys: step c, lane half h, token: 16 bytes at ((block * C + c) * 64 + 32 h + token) * 16; values: run a of 32
        // channels, 16 tokens s, lane half h, channel: ((block * A + a) * 2 + s) * 64 + 32 h + channel % 32
        int ref_new = ref;
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (cur.unit[i] >= 0) ref_new = __builtin_amdgcn_readfirstlane(cur.vb[i]) > ref_new ? __builtin_amdgcn_readfirstlane(cur.vb[i]) : ref_new;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int at = (threadIdx.x + 256 * i) * 16, blk = at / (32 * D), in = at % (32 * D);
            const int token = in / D, c = in % D / 16;
            *reinterpret_cast<kv_f16x8 *>(kt + (((blk * C + c) * 64) + token) * 16) = kv_f16_of(cur.k[i].x, cur.k[i].y, 1.f);
            *reinterpret_cast<kv_f16x8 *>(kt + (((blk * C + c) * 64) + 32 + token) * 16) = kv_f16_of(cur.k[i].z, cur.k[i].w, 1.f);
            const int a = in / 1024, d16 = in / 64 % 16, g = in / 16 % 4, s = g >> 1, h = g & 1;
            const bool named = (blk ? cur.unit[1] : cur.unit[0]) >= 0;
            const float vf = kv_pow2((blk ? cur.vb[1] : cur.vb[0]) - ref_new);
            uint4 w = cur.v[i];
            if (key + kTileKeys > len || !named) {      // codes of tokens that do not exist
                uint32_t live[2] = {0u, 0u};
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (named && key + 32 * blk + kv_slot_token(g) + (j & 3) + 8 * (j >> 2) < len) live[j >> 2] |= 0xffu << (8 * (j & 3));
                w.x &= live[0]; w.y &= live[1]; w.z &= live[0]; w.w &= live[1];
            }
            unsigned char *dst = vt + (((blk * A + a) * 2 + s) * 64 + 32 * h + d16) * 16;
            *reinterpret_cast<kv_f16x8 *>(dst) = kv_f16_of(w.x, w.y, vf);
            *reinterpret_cast<kv_f16x8 *>(dst + 256) = kv_f16_of(w.z, w.w, vf);
        }
        const long long unit[2] = {cur.unit[0], cur.unit[1]};
        const float kf[2] = {to_t * kv_pow2(cur.kb[0] - 127), to_t * kv_pow2(cur.kb[1] - 127)};
        __syncthreads();
        if (key + kTileKeys < wg_hi) cur = load(key + kTileKeys);
        if (ref_new != ref) {
            const float f = kv_pow2(ref - ref_new);
#pragma unroll
            for (int a = 0; a < A; ++a) o[a] *= f;
            ref = ref_new;
        }
        if (key >= any_hi || key + kTileKeys <= any_lo) continue;      // (of no row of this wavefront)

        kv_floatx16 s[2] = {};
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 2; ++i)
                s[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const kv_f16x8 *>(kt + ((i * C + c) * 64 + lane) * 16), qf[c], s[i], 0, 0, 0);
        const bool edge = unit[0] < 0 || unit[1] < 0 || key < all_lo || key + kTileKeys > all_hi;
        if (edge) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const int at = key + 32 * i + 8 * (v >> 2) + 4 * h32 + (v & 3);
                    const bool ok = unit[i] >= 0 && at >= seen_lo && at < seen_hi && at < len;
                    s[i][v] = ok ? s[i][v] * kf[i] : -__builtin_inff();
                }
        } else {
            s[0] *= kf[0];
            s[1] *= kf[1];
        }
        float top = fmaxf(s[0][0], s[1][0]);
#pragma unroll
        for (int v = 1; v < 16; ++v) top = fmaxf(top, fmaxf(s[0][v], s[1][v]));
        top = kv_max32(top);
        if (__builtin_amdgcn_ballot_w64(top > m + kSlack) != 0ull) {
            const float m_new = fmaxf(m, top), keep = __builtin_amdgcn_exp2f(m - m_new);
            l *= keep;
#pragma unroll
            for (int a = 0; a < A; ++a) o[a] *= keep;
            m = m_new;
        }
        const float base = m - kShift;
        kv_f16x8 pf[4];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const float e = __builtin_amdgcn_exp2f(s[i][v] - base);
                l += e;
                pf[2 * i + v / 8][v % 8] = (_Float16)e;
            }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int a = 0; a < A; ++a)
                o[a] = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const kv_f16x8 *>(vt + ((((i / 2) * A + a) * 2 + i % 2) * 64 + lane) * 16), pf[i], o[a], 0, 0, 0);
    }

    l = kv_sum32(l);
    if (row0 + wave * 32 + l32 >= rows) return;
    const float inv = (l > 0.f ? 1.f / l : l == l ? 0.f : l) * kv_pow2(ref - 127);      // (no key seen: zeros)
    uint16_t *dst = p.out + ((size_t)(t0 + tok) * p.q_heads + qh) * D;
#pragma unroll
    for (int a = 0; a < A; ++a)
#pragma unroll
        for (int v = 0; v < 16; v += 4) {
            const kv_bf16x2 lo = {(__bf16)(o[a][v] * inv), (__bf16)(o[a][v + 1] * inv)}, hi = {(__bf16)(o[a][v + 2] * inv), (__bf16)(o[a][v + 3] * inv)};
            *reinterpret_cast<uint2 *>(dst + 32 * a + 2 * v + 4 * h32) = make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
        }
}

}  // namespace

hipError_t launch_kv_attention_tile(const KvAttentionParams &p, hipStream_t stream) {
    const long long items = (long long)p.batch.total * p.group / kTileRows + p.batch.sequences;
    const dim3 grid((uint32_t)(items * p.cache.heads));
    switch (p.cache.dim) {
        case 64: kv_tile_kernel<64><<<grid, 256, 0, stream>>>(p); break;
        case 128: kv_tile_kernel<128><<<grid, 256, 0, stream>>>(p); break;
        case 256: kv_tile_kernel<256><<<grid, 256, 0, stream>>>(p); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

}  // namespace svdq
