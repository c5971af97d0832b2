// Attention of many query rows over the paged 8-bit cache: chunks of prompts, joint attention of all tokens of an image (layout: kv_common.h).
//
//   O_i = sum_j softmax_j(scale q'_i . k_j) v_j,   q' the rotated query, j over the keys that row i sees.
//
// The rows of a sequence and key head are its new tokens times the query heads that share the head, so a tile of keys serves the whole group.  A
// workgroup has 128 rows (four wavefronts, two workgroups on a CU) or 256 (eight, one; head size 128, long even batches), 32 to a wavefront; keys and values go by
// in tiles of 64 tokens, read once per workgroup as codes, converted to f16 on the way into LDS (exact: codes of the keys, code * 2^(byte - reference) of the values, the
// reference exponent the largest so far, while the bytes are at most 15 apart: kv_common.h has the other way) and laid out as operands, so that an operand read is 64 lanes x 16 bytes in a row.  S^T = K Q^T by
// v_mfma_f32_32x32x16_f16: a lane has one row of queries, its accumulators are the operand of O^T = V^T P^T as they stand, and maximum and sum of a row are one exchange
// between lane halves away.  Statistics in fp32; P is exp2(t - m + 8) in f16, at most 2^14 before the maximum is renewed, so weights down to 2^-22 of the
// largest keep eleven bits and those below 2^-33 are zero; Q in f16, scaled by a power of two per row, for the same eleven bits down to 2^-28 of the row's largest.
// The scores of a tile are made beside the weights of the one before, codes are requested two and three tiles ahead, pages and scale bytes 32 tiles ahead; one barrier a tile.
// Few row tiles on many keys take parts of the keys, which kv_meet_kernel joins.  A wavefront whose rows are past the sequence's only carries codes.
// Bound: matrix cores and vector ALU, which overlap little, at the chip's power limit (1.9 of 2.4 GHz under the profiler).  8192 tokens, 32 query heads on 8, on 16384 keys 1540 us, 1.07 PFLOP/s
// (a library product of 8192 cubed in f16 reaches 1.215): matrix cores busy 51 % of the time, vector ALU 55 %; 4608 tokens of 24 heads, all with all, 280 us, 48 and 54 %, and 432
// tiles are two rounds of 256 CUs; six ragged chunks of up to 2111 tokens 350 us, 43 and 58 %; heads of 64, 8192 tokens on 16384 keys 1036 us, 34 and 68 %.  What a workgroup of 128 rows costs beside its tiles (1.05 us each): scan over
// the sequences 1.2 us, queries and first pages 2.2, turning 2.5, first codes 1.4, out 2, of which the other workgroup of the CU covers about two thirds.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <type_traits>

#include "kernels.h"
#include "kv_common.h"
#include "layout.h"
#include "lds_limit.h"

namespace svdq {
namespace {

constexpr float kNone = -3.4028235e38f;          // the running maximum before the first key: the lowest number, so that any score of a key that is seen renews it
constexpr float kShift = 8.f, kSlack = 6.f;      // P is exp2(t - m + kShift); m is renewed when a score passes it by kSlack
constexpr float kFar = 16777216.f;               // exponents past it (2^24) have steps of two and more
constexpr int kTileKeys = 64;

// LDS of a tile of 64 keys as operands: of the keys step c, lane half h, token; of the values run a of 32 channels, slot g, channel.  The pads spread what
// eight neighbouring lanes write over all banks.
constexpr int kStepBytes = 1024 + 16;
constexpr int kSlotBytes = 512 + 32;
constexpr int k_bytes(int D) { return 2 * (D / 16) * kStepBytes; }
constexpr int v_bytes(int D) { return 2 * (D / 32) * 4 * kSlotBytes; }
// or the queries on their way in, or the output's on its way out
constexpr int tile_lds_bytes(int D, int waves) {
    const int tiles = 2 * (k_bytes(D) + v_bytes(D)), queries = waves * (D / 8 * 33 * 16 + 128), out = waves * 32 * (64 * 4 + 16);
    return tiles > queries ? tiles > out ? tiles : out : queries > out ? queries : out;
}

template <int D, int WAVES>
__global__ __launch_bounds__(64 * WAVES, D > 128 ? 1 : 2) void kv_tile_kernel(KvAttentionParams p) {
    constexpr int C = D / 16, A = D / 32, kRows = 32 * WAVES, kThreads = 64 * WAVES;
    constexpr int N = kTileKeys * D / (kThreads * 16);      // 16-byte pieces of a tile of codes per thread: 1, 2, 4
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l32 = lane & 31, h32 = lane >> 5;
    const int head = blockIdx.x % p.cache.heads, part = blockIdx.y;
    const KvItem item = kv_item(p.batch, blockIdx.x / p.cache.heads, [&](int n, int) { return n * p.group < p.least_rows ? 0 : (n * p.group + kRows - 1) / kRows; });
    const int b = item.sequence, local = item.local, t0 = item.first, n = item.count;
    const int len = kv_length(p.cache, p.batch, item.value), rows = n * p.group, tiles = (rows + kRows - 1) / kRows;
    if (local < 0 || local >= tiles) return;
    const int row0 = (p.causal ? tiles - 1 - local : local) * kRows;      // (causal: the rows with the most keys first)
    auto hi_of = [&](int at) { return at < 0 ? 0 : p.causal ? at + 1 : len; };      // (a token without a position sees nothing)
    auto lo_of = [&](int at) { return p.causal && p.window > 0 && at + 1 > p.window ? at + 1 - p.window : 0; };
    auto pos_of = [&](int row) { return len - n + (row < rows ? row : rows - 1) / p.group; };
    // keys that some row of the workgroup sees, and those that all rows of the wavefront see
    const int wg_lo = lo_of(pos_of(row0)), wg_hi = hi_of(pos_of(row0 + kRows - 1));
    const int w_first = pos_of(row0 + wave * 32), w_last = pos_of(row0 + wave * 32 + 31);
    const int all_lo = lo_of(w_last), all_hi = hi_of(w_first);
    const bool idle = row0 + wave * 32 >= rows;      // no row is left for the wavefront: it brings codes to LDS, and leaves its SIMD to the others
    // tiles of keys, and this part's share of them
    const int key_a = wg_lo / kTileKeys * kTileKeys, tiles_a = wg_hi > key_a ? (wg_hi - key_a + kTileKeys - 1) / kTileKeys : 0;
    const int tile0 = (int)((long long)tiles_a * part / p.parts), tiles_k = (int)((long long)tiles_a * (part + 1) / p.parts) - tile0;
    const int key0 = key_a + tile0 * kTileKeys;

    // ---- the way of the codes: pages and scale bytes of 64 blocks (32 tiles) at a time, one in a lane; codes by way of registers ----
    const int32_t *table = p.batch.table + (size_t)b * p.batch.table_width;
    const int bs = p.cache.page_shift - 5, blk0 = key0 >> 5, blk_z = (wg_hi + 31) >> 5, blk1 = blk_z < blk0 + 2 * tiles_k ? blk_z : blk0 + 2 * tiles_k;
    // (a unit is a block of a head, 2 KB of codes at least: 32 bits count them)
    int unit_l = -1, kb_l = 0, vb_l = 0, unit_a = -1, kb_a = 0, vb_a = 0;      // of the window in use, and of the one after it; -1: no such block
    KvSpread spread;
    bool wide = false;      // the values' scales are too far apart for one reference (the same in all wavefronts)
    auto look_up_pages = [&](int t) {      // t a multiple of 32
        const int blk = blk0 + 2 * t + lane;
        unit_a = blk < blk1 ? table[blk >> bs] : -1;
    };
    auto look_up_bytes = [&](int t) {
        const bool named = (uint32_t)unit_a < (uint32_t)p.cache.pages;
        unit_a = named ? (int)((((uint32_t)unit_a * (uint32_t)p.cache.heads + (uint32_t)head) << bs) + ((blk0 + 2 * t + lane) & ((1 << bs) - 1))) : -1;
        const size_t u = named ? (size_t)(uint32_t)unit_a : 0;
        kb_a = p.cache.ks[u];
        vb_a = p.cache.vs[u];
    };
    auto next_window = [&]() {
        unit_l = unit_a;
        kb_l = kb_a;
        vb_l = unit_a == -1 ? 0 : vb_a;
        wide = wide || spread.add(vb_l);
    };
    // what is known of a tile: its blocks and their scale bytes
    struct Facts { int unit[2], kb[2], vb[2]; };
    auto facts_of = [&](int t) {
        Facts f;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            f.unit[i] = __builtin_amdgcn_readlane(unit_l, 2 * (t & 31) + i);
            f.kb[i] = __builtin_amdgcn_readlane(kb_l, 2 * (t & 31) + i);
            f.vb[i] = __builtin_amdgcn_readlane(vb_l, 2 * (t & 31) + i);
        }
        return f;
    };
    auto named = [](const Facts &f) { return f.unit[0] != -1 && f.unit[1] != -1; };
    auto request = [&](uint4 (&w)[N], const uint8_t *codes, const Facts &f) {      // (no such block: the cache's first)
        const uint8_t *at_blk[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) at_blk[i] = codes + (size_t)(f.unit[i] == -1 ? 0u : (uint32_t)f.unit[i]) * (32 * D);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int at = (threadIdx.x + kThreads * i) * 16, blk = at / (32 * D), in = at % (32 * D);
            w[i] = *reinterpret_cast<const uint4 *>((blk ? at_blk[1] : at_blk[0]) + in);
        }
    };
    // piece i of a tile of codes to operands
    auto keys_to_lds = [&](const uint4 (&w)[N], unsigned char *kt, int i) {
        const int at = (threadIdx.x + kThreads * i) * 16, blk = at / (32 * D), in = at % (32 * D), token = in / D, c = in % D / 16;
        unsigned char *dst = kt + (blk * C + c) * kStepBytes + token * 16;
        *reinterpret_cast<kv_f16x8 *>(dst) = kv_f16_of(w[i].x, w[i].y, 1.f);
        *reinterpret_cast<kv_f16x8 *>(dst + 512) = kv_f16_of(w[i].z, w[i].w, 1.f);
    };
    auto values_to_lds = [&](const uint4 (&w)[N], unsigned char *vt, const Facts &f, int t, int ref, int i, auto partial) {
        const int at = (threadIdx.x + kThreads * i) * 16, blk = at / (32 * D), in = at % (32 * D), a = in / 1024, d16 = in / 64 % 16, g = in / 16 % 4;
        const float vf = blk ? kv_pow2(f.vb[1] - ref) : kv_pow2(f.vb[0] - ref);
        uint32_t live[2] = {~0u, ~0u};      // codes of tokens that exist
        if (decltype(partial)::value) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (key0 + t * kTileKeys + 32 * blk + kv_slot_token(g) + (j & 3) + 8 * (j >> 2) >= len) live[j >> 2] &= ~(0xffu << (8 * (j & 3)));
        }
        unsigned char *dst = vt + ((blk * A + a) * 4 + g) * kSlotBytes + d16 * 16;
        *reinterpret_cast<kv_f16x8 *>(dst) = kv_f16_of(w[i].x & live[0], w[i].y & live[1], vf);
        *reinterpret_cast<kv_f16x8 *>(dst + 256) = kv_f16_of(w[i].z & live[0], w[i].w & live[1], vf);
    };
    auto clear_unnamed = [&](uint4 (&w)[N], const Facts &f) {      // values of blocks that do not exist
        if (named(f)) return;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if ((((int)threadIdx.x + kThreads * i) * 16 / (32 * D) ? f.unit[1] : f.unit[0]) == -1) w[i] = make_uint4(0u, 0u, 0u, 0u);
    };
    const auto kt = [&](int t) { return lds + (t & 1) * k_bytes(D); };
    const auto vt = [&](int t) { return lds + 2 * k_bytes(D) + (t & 1) * v_bytes(D); };

    // ---- the queries: f16 of the rotated row times a power of two that brings its largest element to [2^14, 2^15).  Loaded a unit of 16 channels a lane
    // (the two runs of eight that the rotation pairs), neighbouring lanes with neighbouring channels; each wavefront turns its rows and lays them down in its own part of
    // LDS as operands. ----
    kv_f16x8 qf[C];
    float to_t = 0.f;      // score -> exponent of 2, but for the block's scale; not negative: a negative scale turns the queries' sign
    constexpr int U = D / 16, PER = U < 8 ? U / 2 : 4;      // units of a row, of a lane at a time
    constexpr int kChunk = 33 * 16;         // bytes of a run of eight channels of 32 rows in LDS
    unsigned char *my_queries = lds + wave * (2 * U * kChunk + 128);
    float *factors = reinterpret_cast<float *>(my_queries + 2 * U * kChunk);
    look_up_pages(0);
    if (idle) {
        look_up_bytes(0);
    } else {
        const int half = p.rope.dims / 2;
        for (int i0 = 0; i0 < U / 2; i0 += PER) {
            uint4 own[PER][2];
            float4 c[PER][2], s[PER][2];
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int u = lane + 64 * (i0 + i), row = u / U, pr = u % U;
                const int r = row0 + wave * 32 + row < rows ? row0 + wave * 32 + row : rows - 1;
                const int tok = r / p.group, qh = head * p.group + r % p.group, pos = len - n + tok;
                const uint16_t *src = p.q.data + (size_t)(t0 + tok) * p.q.token_stride + qh * p.q.head_stride;
                const bool halves = !p.rope.interleaved && pr < p.rope.dims / 16;
                own[i][0] = *reinterpret_cast<const uint4 *>(src + (halves ? pr * 8 : pr * 16));
                own[i][1] = *reinterpret_cast<const uint4 *>(src + (halves ? pr * 8 + half : pr * 16 + 8));
                if (pr < p.rope.dims / 16) {
                    const float *t = p.rope.table + (size_t)(pos < 0 ? 0 : pos < p.rope.positions ? pos : p.rope.positions - 1) * p.rope.dims + pr * 8;
                    c[i][0] = *reinterpret_cast<const float4 *>(t);
                    c[i][1] = *reinterpret_cast<const float4 *>(t + 4);
                    s[i][0] = *reinterpret_cast<const float4 *>(t + half);
                    s[i][1] = *reinterpret_cast<const float4 *>(t + half + 4);
                } else {
                    c[i][0] = c[i][1] = s[i][0] = s[i][1] = make_float4(0.f, 0.f, 0.f, 0.f);
                }
            }
            if (i0 == 0) look_up_bytes(0);
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int u = lane + 64 * (i0 + i), row = u / U, pr = u % U;
                const bool turn = pr < p.rope.dims / 16, halves = !p.rope.interleaved && turn;
                float x[2][8];
                kv_floats(own[i][0], x[0]);
                kv_floats(own[i][1], x[1]);
                const float cc[8] = {c[i][0].x, c[i][0].y, c[i][0].z, c[i][0].w, c[i][1].x, c[i][1].y, c[i][1].z, c[i][1].w};
                const float ss[8] = {s[i][0].x, s[i][0].y, s[i][0].z, s[i][0].w, s[i][1].x, s[i][1].y, s[i][1].z, s[i][1].w};
                if (turn) {
                    if (!p.rope.interleaved) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float a = x[0][e], y = x[1][e];
                            x[0][e] = kv_turn_a(a, y, cc[e], ss[e]);
                            x[1][e] = kv_turn_b(a, y, cc[e], ss[e]);
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float a = x[e / 4][2 * (e % 4)], y = x[e / 4][2 * (e % 4) + 1];
                            x[e / 4][2 * (e % 4)] = kv_turn_a(a, y, cc[e], ss[e]);
                            x[e / 4][2 * (e % 4) + 1] = kv_turn_b(a, y, cc[e], ss[e]);
                        }
                    }
                }
                float most = 0.f;      // (NaN if one is NaN)
#pragma unroll
                for (int e = 0; e < 8; ++e) most = __builtin_elementwise_maximum(__builtin_elementwise_maximum(most, __builtin_fabsf(x[0][e])), __builtin_fabsf(x[1][e]));
                const uint32_t top = __float_as_uint(kv_max_lanes<U>(most)) & 0x7fffffffu;      // (the row's units are neighbouring lanes)
                const int e = (int)((top >= 0x7f800000u ? 0x7f800000u : top) >> 23) - 127;      // largest in [2^e, 2^(e + 1))
                const int up = e < -100 ? 114 : e > 127 ? 0 : 14 - e;                           // (not finite: as it is, the row becomes NaN)
                const float f = p.scale < 0.f ? -kv_pow2(up) : kv_pow2(up);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    kv_f16x8 w;
#pragma unroll
                    for (int k = 0; k < 8; ++k) w[k] = (_Float16)(x[j][k] * f);
                    const int chunk = halves ? pr + j * (half / 8) : 2 * pr + j;
                    *reinterpret_cast<kv_f16x8 *>(my_queries + chunk * kChunk + row * 16) = w;
                }
                if (pr == 0) factors[row] = __builtin_fabsf(p.scale) * kv_pow2(-up);
            }
        }
    }
    uint4 kw[2][N], vw[2][N];      // codes on their way: of keys and values of even and odd tiles
    next_window();
    Facts f0 = facts_of(0), f1 = facts_of(1), f2 = facts_of(2), f3 = facts_of(3), f4 = facts_of(4);      // of tiles t .. t + 4
    if (tiles_k > 0 && !wide) {
        request(kw[0], p.cache.k, f0);
        request(vw[0], p.cache.v, f0);
        request(kw[1], p.cache.k, f1);
        request(vw[1], p.cache.v, f1);
    }
    if (!idle) {
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int c = 0; c < C; ++c) qf[c] = *reinterpret_cast<const kv_f16x8 *>(my_queries + (2 * c + h32) * kChunk + l32 * 16);      // step c: channels 16 c + 8 h32 .. + 7
        to_t = factors[l32];
    }
    kv_lds_barrier();      // (the tiles go where the queries lie)

    kv_floatx16 o[A] = {};
    float m = kNone, l = 0.f;
    int ref = 0;                   // byte of the reference scale of the values in o
    float kf[2];                   // factors of the scores that weight_pair() takes
    bool far = false;              // a row's maximum is past kFar, or was
    float base;                    // kShift - m; kShift where the scores have lost m already
    kv_f16x8 pf[4];
    typedef kv_floatx16 Scores[2];

    auto key_operand = [&](const unsigned char *tile, int c, int i) { return *reinterpret_cast<const kv_f16x8 *>(tile + (i * C + c) * kStepBytes + lane * 16); };
    auto value_operand = [&](const unsigned char *tile, int k) {      // product k: 16 tokens k / A, run k % A of channels
        return *reinterpret_cast<const kv_f16x8 *>(tile + (((k / A / 2) * A + k % A) * 4 + 2 * (k / A % 2) + h32) * kSlotBytes + l32 * 16);
    };
    auto add_values = [&](kv_f16x8 w, int k) { o[k % A] = __builtin_amdgcn_mfma_f32_32x32x16_f16(w, pf[k / A], o[k % A], 0, 0, 0); };
    // maximum of half a block's scores, on top of `x` (NaN if one is NaN: the row is NaN then, whatever its maximum)
    auto largest_half = [&](float x, const kv_floatx16 &s, int half) {
#pragma unroll
        for (int v = 8 * half; v < 8 * half + 8; v += 2) x = __builtin_elementwise_maximum(__builtin_elementwise_maximum(x, s[v]), s[v + 1]);
        return x;
    };
    auto largest = [&](const Scores &s, float (&top)[2]) {
#pragma unroll
        for (int i = 0; i < 2; ++i) top[i] = largest_half(largest_half(-__builtin_inff(), s[i], 0), s[i], 1);
    };
    // masks the scores of tile t and renews the maximum if they pass it; top: largest(s)
    auto look_at = [&](Scores &s, float (&top)[2], const Facts &f, int t) {
        const int key = key0 + t * kTileKeys;
        if (!named(f) || key < all_lo || key + kTileKeys > all_hi) {
            const int pos = pos_of(row0 + wave * 32 + l32), seen_hi = hi_of(pos) < len ? hi_of(pos) : len, seen_lo = lo_of(pos);
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const int at = key + 32 * i + 8 * (v >> 2) + 4 * h32 + (v & 3);
                    s[i][v] = f.unit[i] != -1 && at >= seen_lo && at < seen_hi ? s[i][v] : -__builtin_inff();
                }
            largest(s, top);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {      // (not zero, so that what is masked stays masked; not infinite, so that a sum of zero is a score of zero)
            kf[i] = kv_within_range(to_t * kv_pow2(f.kb[i] - 127));
            kf[i] = kf[i] < 1.1754944e-38f ? 1.1754944e-38f : kf[i];
        }
        const float most = kv_max32(__builtin_elementwise_maximum(top[0] * kf[0], top[1] * kf[1]));
        if (__builtin_amdgcn_ballot_w64(most > m + kSlack) != 0ull) {
            const float m_new = fmaxf(m, most), keep = __builtin_amdgcn_exp2f(m - m_new);
            l *= keep;
#pragma unroll
            for (int a = 0; a < A; ++a) o[a] *= keep;
            m = m_new;
            far = far || __builtin_amdgcn_ballot_w64(!(__builtin_fabsf(m) <= kFar) && most != -__builtin_inff()) != 0ull;
        }
        base = kShift - m;
        // weight_pair() adds m to the product before it is rounded, but m is a rounded product, and kShift is lost beside a large one: once a maximum is far out, scores
        // become their rounded distances to it here, so that the largest is zero as it should be (and NaN where it passed fp32)
        if (far) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
#pragma unroll
                for (int v = 0; v < 16; ++v) s[i][v] = s[i][v] * kf[i] - m;
                kf[i] = 1.f;
            }
            base = kShift;
        }
    };
    auto weight_pair = [&](const Scores &s, int q) {      // pair q of 16: two weights, and their sum
        const int i = q / 8, v = 2 * (q % 8);
        const kv_f16x2 e = {(_Float16)__builtin_amdgcn_exp2f(__builtin_fmaf(s[i][v], kf[i], base)), (_Float16)__builtin_amdgcn_exp2f(__builtin_fmaf(s[i][v + 1], kf[i], base))};
        l = __builtin_amdgcn_fdot2(e, kv_f16x2{(_Float16)1.f, (_Float16)1.f}, l, false);      // (the sum of what is multiplied)
        pf[2 * i + v / 8][v % 8] = e[0];
        pf[2 * i + v / 8][v % 8 + 1] = e[1];
    };
    auto refer = [&](const Facts &f) { return f.vb[0] > f.vb[1] ? f.vb[0] : f.vb[1]; };
    auto grow = [&](int to) {      // the reference scale
        if (to <= ref) return;
        const float f = kv_pow2(ref - to);
#pragma unroll
        for (int a = 0; a < A; ++a) o[a] *= f;
        ref = to;
    };

    // Tile t + 1's scores are made beside tile t's weights; in LDS the keys are a tile ahead of the values:
    //   step t: S(t + 1) from keys t + 1, P(t) from S(t), O += P(t) V(t); keys t + 2 and values t + 1 go to LDS, keys t + 4 and values t + 3 are requested
    auto advance = [&](int far) {      // facts of the next step: tile `far` comes in
        if ((far & 7) == 0) {
            if ((far & 31) == 8) look_up_pages(far + 24);
            else if ((far & 31) == 16) look_up_bytes(far + 16);
            else if ((far & 31) == 0) next_window();
        }
        f1 = f2;
        f2 = f3;
        f3 = f4;
        f4 = facts_of(far);
    };
    // (a window of pages that turns out too wide ends both loops below at the same step: it is one of tiles that are still to come, four at least)
    const bool ordinary = tiles_k > 0 && !wide;
    if (ordinary) {
        ref = refer(f0);
        clear_unnamed(vw[0], f0);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            keys_to_lds(kw[0], kt(0), i);
            values_to_lds(vw[0], vt(0), f0, 0, ref, i, std::true_type{});
        }
        request(kw[0], p.cache.k, f2);
        request(vw[0], p.cache.v, f2);
#pragma unroll
        for (int i = 0; i < N; ++i) keys_to_lds(kw[1], kt(1), i);
        request(kw[1], p.cache.k, f3);
        kv_lds_barrier();
    }
    if (ordinary && idle) {      // a wavefront's part of the steps but for its products
        kv_lds_barrier();
        auto carry = [&](uint4 (&kn)[N], uint4 (&vn)[N], int t) {
            ref = refer(f1) > ref ? refer(f1) : ref;
            clear_unnamed(vn, f1);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                values_to_lds(vn, vt(t + 1), f1, t + 1, ref, i, std::true_type{});
                keys_to_lds(kn, kt(t), i);
            }
            request(vn, p.cache.v, f3);
            request(kn, p.cache.k, f4);
            kv_lds_barrier();
            advance(t + 5);
        };
        for (int t = 0; t + 1 < tiles_k && !wide; t += 2) {
            carry(kw[0], vw[1], t);
            if (t + 2 < tiles_k) carry(kw[1], vw[0], t + 1);
        }
    } else if (ordinary) {
        Scores even, odd;
        float top[2];
        even[0] = even[1] = kv_floatx16{};
#pragma unroll
        for (int k = 0; k < 2 * C; ++k) even[k & 1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(key_operand(kt(0), k / 2, k & 1), qf[k / 2], even[k & 1], 0, 0, 0);
        largest(even, top);
        look_at(even, top, f0, 0);
        kv_lds_barrier();             // (step 0 puts keys 2 in the place of keys 0)
        // The order within a step is fixed by hand: operands are read ahead of their products.  Four wavefronts (two workgroups on a CU, which drift apart): a product is
        // issued and the vector work of its length follows.  Eight (one workgroup): the products of the scores by themselves, at a higher priority, so that one
        // wavefront of a SIMD multiplies while the other makes weights; mixed 1560 us, apart 1527 (8192 rows x 4 heads on 16384 keys), and four wavefronts 1596
        // mixed, 1645 apart.
        constexpr bool APART = WAVES == 8;
        auto step = [&](Scores &now, Scores &next, uint4 (&kn)[N], uint4 (&vn)[N], int t, auto partial) {      // kn: keys t + 2, vn: values t + 1
            const int held = refer(f1) > ref ? refer(f1) : ref;      // the scale that the next values in LDS refer to
            const unsigned char *keys = kt(t + 1), *values = vt(t);
            clear_unnamed(vn, f1);
            if (APART) __builtin_amdgcn_s_setprio(1);
            kv_f16x8 kop[2][2], vop[4];
#pragma unroll
            for (int i = 0; i < 2; ++i) kop[0][i] = key_operand(keys, 0, i);
            next[0] = next[1] = kv_floatx16{};
#pragma unroll
            for (int c = 0; c < C; ++c) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if (c + 1 < C) kop[(c + 1) & 1][i] = key_operand(keys, c + 1, i);
                    else vop[i] = value_operand(values, i);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) next[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kop[c & 1][i], qf[c], next[i], 0, 0, 0);
                if (!APART) {
#pragma unroll
                    for (int q = 16 * c / C; q < 16 * (c + 1) / C; ++q) weight_pair(now, q);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            if (APART) {
                __builtin_amdgcn_s_setprio(0);
#pragma unroll
                for (int q = 0; q < 16; ++q) weight_pair(now, q);
                __builtin_amdgcn_sched_barrier(0);
            }
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int k = 0; k < 4 * A; ++k) {
                if (k + 2 < 4 * A) vop[(k + 2) & 3] = value_operand(values, k + 2);
                add_values(vop[k & 3], k);
                if (k % A == 0) {
                    const int i = k / A;      // of four
                    top[i / 2] = largest_half(i % 2 ? top[i / 2] : -__builtin_inff(), next[i / 2], i % 2);
                }
#pragma unroll
                for (int i = 2 * N * k / (4 * A); i < 2 * N * (k + 1) / (4 * A); ++i) {      // 2 N pieces
                    if (i < N) values_to_lds(vn, vt(t + 1), f1, t + 1, held, i, partial);
                    else keys_to_lds(kn, kt(t), i - N);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            __builtin_amdgcn_s_setprio(0);
            request(vn, p.cache.v, f3);
            request(kn, p.cache.k, f4);
            grow(held);
            look_at(next, top, f1, t + 1);
            kv_lds_barrier();
            advance(t + 5);
        };
        int t = 0;
        for (; t + 4 <= tiles_k && !wide; t += 2) {      // (the last tile's values may be partial: step tiles_k - 2)
            step(even, odd, kw[0], vw[1], t, std::false_type{});
            step(odd, even, kw[1], vw[0], t + 1, std::false_type{});
        }
        if (!wide) {      // one to three tiles are left, the first one's scores in `even`
            if (t + 1 < tiles_k) {
                step(even, odd, kw[0], vw[1], t, std::true_type{});
                ++t;
                if (t + 1 < tiles_k) {
                    step(odd, even, kw[1], vw[0], t, std::true_type{});
                    ++t;
                } else {
                    even[0] = odd[0];
                    even[1] = odd[1];
                }
            }
#pragma unroll
            for (int q = 0; q < 16; ++q) weight_pair(even, q);
#pragma unroll
            for (int k = 0; k < 4 * A; ++k) add_values(value_operand(vt(t), k), k);
        }
    }
    int row_ref = ref;
    if (__builtin_expect(wide && !idle, 0)) {      // from the start, a block at a time, each wavefront by itself
#pragma unroll
        for (int a = 0; a < A; ++a) o[a] = kv_floatx16{};
        m = kNone;
        l = 0.f;
        row_ref = 0;
        const int pos = pos_of(row0 + wave * 32 + l32), seen_hi = hi_of(pos) < len ? hi_of(pos) : len, seen_lo = lo_of(pos);
        for (int blk = blk0; blk < blk1; ++blk) {
            const long long unit = kv_unit(p.cache, p.batch.table, p.batch.table_width, b, head, blk);
            if (unit < 0) continue;
            const uint8_t *k = p.cache.k + (size_t)unit * (32 * D) + l32 * D + 8 * h32, *v = p.cache.v + (size_t)unit * (32 * D) + (l32 % 16 * 4 + h32) * 16 + l32 / 16 * 8;
            kv_floatx16 s = {};
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const uint2 w = *reinterpret_cast<const uint2 *>(k + 16 * c);
                s = __builtin_amdgcn_mfma_f32_32x32x16_f16(kv_f16_of(w.x, w.y, 1.f), qf[c], s, 0, 0, 0);
            }
            const float f = kv_within_range(to_t * kv_pow2((int)p.cache.ks[unit] - 127));
            float top = -__builtin_inff();
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int at = blk * kKvBlock + 8 * (i >> 2) + 4 * h32 + (i & 3);
                s[i] = at >= seen_lo && at < seen_hi ? s[i] * f : -__builtin_inff();
                top = fmaxf(top, s[i]);
            }
            top = kv_max32(top);
            const float from = top > -__builtin_inff() ? top : 0.f;
            float sum = 0.f, largest_o = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const _Float16 e = (_Float16)__builtin_amdgcn_exp2f(s[i] - from + kShift);
                sum += (float)e;
                pf[i / 8][i % 8] = e;
            }
#pragma unroll
            for (int a = 0; a < A; ++a)
#pragma unroll
                for (int i = 0; i < 16; ++i) largest_o = fmaxf(largest_o, __builtin_fabsf(o[a][i]));
            const KvJoin join = kv_join(m, row_ref, top, (int)p.cache.vs[unit], kv_max32(largest_o));
            l = l * join.keep_l + sum * join.add_l;
#pragma unroll
            for (int a = 0; a < A; ++a) {
                kv_floatx16 x = {};
#pragma unroll
                for (int g = 0; g < 2; ++g) {      // the lane's slot is 2 g + h32
                    uint2 w = *reinterpret_cast<const uint2 *>(v + a * 1024 + g * 32);
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (blk * kKvBlock + kv_slot_token(2 * g + h32) + (j & 3) + 8 * (j >> 2) >= len) (j < 4 ? w.x : w.y) &= ~(0xffu << (8 * (j & 3)));
                    x = __builtin_amdgcn_mfma_f32_32x32x16_f16(kv_f16_of(w.x, w.y, 1.f), pf[g], x, 0, 0, 0);
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) o[a][i] = __builtin_amdgcn_ldexpf(o[a][i] * join.keep, join.keep_e) + __builtin_amdgcn_ldexpf(x[i] * join.add, join.add_e);
            }
        }
    }

    // ---- the way out: 32 rows x kOut channels at a time through the wavefront's part of LDS, so that a store writes whole rows ----
    const float sum = kv_sum32(l);
    const bool parts = p.parts > 1;
    const float inv = kv_inverse(sum);
    const auto mean = [&](float x) { return __builtin_amdgcn_ldexpf(x * inv, row_ref - 127); };
    const size_t out_rows = (size_t)p.batch.total * p.q_heads;
    auto out_row = [&](int r) { return (size_t)(t0 + r / p.group) * p.q_heads + head * p.group + r % p.group; };
    const int r_lane = row0 + wave * 32 + l32;
    if (parts) {      // weighted means [part][row][D] and [part][row][2], to be joined by kv_meet_kernel
        if (h32 == 0 && r_lane < rows) *reinterpret_cast<float2 *>(p.part_ml + (part * out_rows + out_row(r_lane)) * 2) = make_float2(m, sum);
        if (tiles_k == 0) return;
    }
    kv_lds_barrier();      // (the last tiles are read)
    if (idle) return;
    constexpr int kOut = 64, kOutRow = kOut * 4 + 16;      // channels of a round and bytes of a row, fp32
    unsigned char *my_rows = lds + wave * 32 * kOutRow;
#pragma unroll
    for (int a0 = 0; a0 < A; a0 += 2) {
#pragma unroll
        for (int a = a0; a < a0 + 2; ++a)
#pragma unroll
            for (int v = 0; v < 16; v += 4)
                *reinterpret_cast<float4 *>(my_rows + l32 * kOutRow + (32 * (a - a0) + 2 * v + 4 * h32) * 4) = make_float4(mean(o[a][v]), mean(o[a][v + 1]), mean(o[a][v + 2]), mean(o[a][v + 3]));
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < 4; ++i) {      // eight channels a lane, eight rows a time
            const int row = 8 * i + lane / 8, d = lane % 8 * 8, r = row0 + wave * 32 + row;
            const float4 x = *reinterpret_cast<const float4 *>(my_rows + row * kOutRow + d * 4), y = *reinterpret_cast<const float4 *>(my_rows + row * kOutRow + d * 4 + 16);
            if (r >= rows) continue;
            if (parts) {
                float *dst = p.partial + (part * out_rows + out_row(r)) * D + 32 * a0 + d;
                *reinterpret_cast<float4 *>(dst) = x;
                *reinterpret_cast<float4 *>(dst + 4) = y;
            } else {
                const kv_bf16x2 w[4] = {{(__bf16)x.x, (__bf16)x.y}, {(__bf16)x.z, (__bf16)x.w}, {(__bf16)y.x, (__bf16)y.y}, {(__bf16)y.z, (__bf16)y.w}};
                *reinterpret_cast<uint4 *>(p.out + out_row(r) * D + 32 * a0 + d) =
                    make_uint4(__builtin_bit_cast(uint32_t, w[0]), __builtin_bit_cast(uint32_t, w[1]), __builtin_bit_cast(uint32_t, w[2]), __builtin_bit_cast(uint32_t, w[3]));
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// Joins the parts of every row in order: each is a weighted mean of values, and they are weighted with their share of the weights, so nothing passes a range that
// the values keep.  A thread has four channels of a row.
template <int D>
__global__ __launch_bounds__(256) void kv_meet_kernel(KvAttentionParams p) {
    constexpr int kRows = 256 / (D / 4);      // rows of a workgroup
    const int row_in = threadIdx.x / (D / 4), d = threadIdx.x % (D / 4) * 4;
    const size_t rows = (size_t)p.batch.total * p.q_heads, row = (size_t)blockIdx.x * kRows + row_in;
    // (tokens of no sequence have no parts)
    int first = p.batch.cu[0], last = p.batch.cu[p.batch.sequences];
    first = first < 0 ? 0 : first;
    last = last > p.batch.total ? p.batch.total : last;
    const long long token = (long long)(row / p.q_heads);
    if (row >= rows || token < first || token >= last) return;
    float2 ml[kKvMostParts];
    float most = kNone, sum = 0.f;
#pragma unroll
    for (int i = 0; i < kKvMostParts; ++i) ml[i] = i < p.parts ? *reinterpret_cast<const float2 *>(p.part_ml + ((size_t)i * rows + row) * 2) : make_float2(kNone, 0.f);
#pragma unroll
    for (int i = 0; i < kKvMostParts; ++i) most = fmaxf(most, ml[i].x);
#pragma unroll
    for (int i = 0; i < kKvMostParts; ++i) {
        ml[i].y *= __builtin_amdgcn_exp2f(ml[i].x - most);
        sum += ml[i].y;
    }
    const float inv = kv_inverse(sum);
    kv_floatx4 x = {};
#pragma unroll
    for (int i = 0; i < kKvMostParts; ++i)
        if (ml[i].y != 0.f) x += *reinterpret_cast<const kv_floatx4 *>(p.partial + ((size_t)i * rows + row) * D + d) * (ml[i].y * inv);      // (a part that saw no key holds no mean)
    const kv_bf16x2 lo = {(__bf16)x[0], (__bf16)x[1]}, hi = {(__bf16)x[2], (__bf16)x[3]};
    *reinterpret_cast<uint2 *>(p.out + row * D + d) = make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
}

template <int D, int WAVES>
hipError_t launch_tile(const KvAttentionParams &p, hipStream_t stream) {
    static LdsLimit limit;
    constexpr int bytes = tile_lds_bytes(D, WAVES);
    if (bytes > 65536) {
        const hipError_t e = limit.raise(reinterpret_cast<const void *>(kv_tile_kernel<D, WAVES>), bytes);
        if (e != hipSuccess) return e;
    }
    const long long items = (long long)p.batch.total * p.group / (32 * WAVES) + p.batch.sequences;
    kv_tile_kernel<D, WAVES><<<dim3((uint32_t)(items * p.cache.heads), p.parts), 64 * WAVES, bytes, stream>>>(p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.parts == 1) return e;
    const size_t rows = (size_t)p.batch.total * p.q_heads;
    constexpr int per = 256 / (D / 4);
    kv_meet_kernel<D><<<(uint32_t)((rows + per - 1) / per), 256, 0, stream>>>(p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_attention_tile(const KvAttentionParams &p, hipStream_t stream) {
    switch (p.cache.dim) {
        case 64: return launch_tile<64, 4>(p, stream);
        case 128: return p.tile_rows == 256 ? launch_tile<128, 8>(p, stream) : launch_tile<128, 4>(p, stream);
        case 256: return launch_tile<256, 4>(p, stream);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace svdq
