// Attention of few query rows over the paged 8-bit cache: the steps of a serving loop (layout: kv_common.h).
//
//   O_i = sum_j softmax_j(scale q'_i . k_j) v_j,   q' the rotated query, j over the keys that row i sees.
//
// The rows of a sequence and key head are its new tokens times the query heads that share the head; sixteen of them are one operand.  Keys are cut into
// chunks, a workgroup of four wavefronts has one chunk of one head, a wavefront takes every fourth block of 32 tokens: S^T = K Q^T by
// v_mfma_f32_16x16x32_f16 with the codes of the keys as exact f16 numbers (rows of the operand: tokens, in an order that makes the accumulators of
// two such products the operand of the next), the block's scale in one factor per row; running maximum and sum per row in fp32; P^T in f16;
// O^T += V^T P^T with the values as code * 2^(byte - reference), the reference exponent the largest so far, which is exact while the wavefront's bytes are at most
// 15 apart (kv_common.h has the other way).  P is scaled by 2^8 (and may reach 2^14
// before the maximum is renewed), so that f16 keeps eleven bits of weights down to 2^-22 of the largest (those below 2^-33 are zero); f16 for Q, scaled by a power of two per
// row, for the same eleven bits down to 2^-28 of the row's largest.
// Loads: the pages and scale bytes of a wavefront's next 64 blocks are looked up at once, one in a lane; the codes of two blocks are in flight (16 KB a
// wavefront, three workgroups a CU), each requested right behind the last use of its registers.
// The wavefronts meet in LDS, as weighted means.  With several chunks the parts lie in the workspace, past the L2s, and the workgroup that finds all of its row tile
// arrived joins them in chunk order (the same bits whoever it is), eight requests in flight a thread; nothing waits for another workgroup.
// First tokens that stay visible before a window are blocks before the window's: the chunks count on over the gap, which is not read.
// Bound: memory, one byte per channel of a key and a value: one sequence of 131071 keys, 8 key heads of 128, 32 query heads 54 us (5.0 TB/s), 64 sequences
// of 100 to 16384 keys 245 us (4.65 TB/s); of 100 to 32768 in a window of 8192 with 64 first tokens and normalised queries 195 us (4.83 TB/s, 193 without either).  A norm alone, without a window,
// adds 0.3 % there (231.3 us and 232.0, the last-level cache holding a part) and 0.6 us to a short call (777 keys 9.6 and 10.2).  Short ones by a chain of round trips: 5.7 us for one block (lengths, table, codes, queries turned on the way), 9.3 us for 777 keys of eight
// heads, where the eight CUs draw 52 GB/s each; 11.4 for 1024 keys and four first tokens, normalised queries, in five pieces (10.9 without).  Eight wavefronts a workgroup gain nothing: 13.0.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <type_traits>

#include "buffer.h"
#include "kernels.h"
#include "kv_common.h"
#include "layout.h"
#include "lds_limit.h"

namespace svdq {
namespace {

constexpr float kNone = -3.4028235e38f;          // the running maximum before the first key: the lowest number, so that any score of a key that is seen renews it
constexpr float kShift = 8.f, kSlack = 6.f;      // P is exp2(t - m + kShift); m is renewed when a score passes it by kSlack
constexpr int WAVES = 4;

template <int D>
struct Block { uint4 k[2][D / 64]; uint4 v[D / 32]; };      // 32 tokens of a head, as a lane holds them

// floats of a row in LDS, and the bytes of a workgroup's LDS: first the queries as operands in fp32 and maxima (and sums of squares) per wavefront, then [wave][row][row_floats] and maximum and sum
// [wave][16][2], or, where parts meet, weights [chunk][row] and 16 bytes a thread
constexpr int row_floats(int D) { return D + 4; }
constexpr int rows_lds_bytes(int D, int waves, int cap, int chunks, bool norm) {
    const int loop = (waves * cap * row_floats(D) + waves * 32) * 4, queries = (D / 32 * 512 + waves * (norm ? 192 : 64)) * 4, parts = chunks > 1 ? (chunks * cap + 4) * 4 + waves * 64 * 16 : 0;
    return loop > parts ? loop > queries ? loop : queries : parts > queries ? parts : queries;
}
constexpr int kAgent = 16;      // cache policy of a buffer access that all XCDs see

// As KvRotating, of a row that is normalised first.  The factor r of the norm is the same for all channels of a row, so it waits: what is turned is x w 2^-32 (which no finite x takes past
// fp32 with weights up to 2^32), and r 2^32 goes into the row's factor of the scores, when the wavefronts' sums of squares have met beside their maxima.
// Every load is made whatever the call needs (from `any`, 32 D bytes that may be read, where there is nothing else), so that no branch lies between the block table's entry, which
// is waited for next, and what was asked for behind it.
constexpr float kHeld = 2.3283064365386963e-10f;      // 2^-32
template <int N>
struct KvReadying {
    uint4 own[N], other[N];
    float c[N][8], s[N][8], w[N][8], w_other[N][8];
    bool ones;
    template <typename Place>
    __device__ __forceinline__ void request(const uint16_t *row, const KvNorm &norm, const KvRope &rope, int pos, int head, Place place, const uint8_t *any) {
        const float *spare = reinterpret_cast<const float *>(any), *weights = kv_norm_row(norm, pos, head);
        const float *t = rope.dims ? rope.table + (size_t)(pos < 0 ? 0 : pos < rope.positions ? pos : rope.positions - 1) * rope.dims : spare;
        const int half = rope.dims / 2;
        ones = weights == nullptr;
        weights = ones ? spare : weights;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int d = place(i) < rope.dims ? place(i) : 0;
            const int first = rope.interleaved ? d / 2 : d >= half ? d - half : d, more = rope.interleaved ? 0 : 4;      // (interleaved: the first four of each)
            const int partner = d >= half ? d - half : d + half;
            own[i] = *reinterpret_cast<const uint4 *>(row + place(i));
            other[i] = *reinterpret_cast<const uint4 *>(row + partner);
            kv_load8(weights + place(i), w[i]);
            kv_load8(weights + partner, w_other[i]);
            const kv_floatx4 a = *reinterpret_cast<const kv_floatx4 *>(t + first), b = *reinterpret_cast<const kv_floatx4 *>(t + first + more);
            const kv_floatx4 e = *reinterpret_cast<const kv_floatx4 *>(t + half + first), f = *reinterpret_cast<const kv_floatx4 *>(t + half + first + more);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                c[i][k] = a[k]; c[i][4 + k] = b[k];
                s[i][k] = e[k]; s[i][4 + k] = f[k];
            }
        }
    }
    // sum, tiny: of the squares of run i's numbers, and of 2^-72 times them
    __device__ __forceinline__ void add_squares(int i, float &sum, float &tiny) const {
        float y[8];
        kv_floats(own[i], y);
        sum += kv_squares(y);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] *= kKvTiny;
        tiny += kv_squares(y);
    }
    template <typename Place>
    __device__ __forceinline__ void finish(const KvRope &rope, Place place, float (&x)[N][8]) const {
        const auto ready = [&](const uint4 &raw, const float (&weight)[8], float (&y)[8]) {
            kv_floats(raw, y);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] *= ones ? kHeld : weight[e] * kHeld;
        };
#pragma unroll
        for (int i = 0; i < N; ++i) ready(own[i], w[i], x[i]);
        if (rope.dims == 0) return;
        const int half = rope.dims / 2;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const bool turn = place(i) < rope.dims, second = place(i) >= half;
            if (rope.interleaved) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float a = x[i][2 * e], b = x[i][2 * e + 1];
                    x[i][2 * e] = turn ? kv_turn_a(a, b, c[i][e], s[i][e]) : a;
                    x[i][2 * e + 1] = turn ? kv_turn_b(a, b, c[i][e], s[i][e]) : b;
                }
            } else {
                float y[8];
                ready(other[i], w_other[i], y);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float z = second ? kv_turn_b(y[e], x[i][e], c[i][e], s[i][e]) : kv_turn_a(x[i][e], y[e], c[i][e], s[i][e]);
                    x[i][e] = turn ? z : x[i][e];
                }
            }
        }
    }
};

// Of a launch: kPlain has neither a norm of the queries nor first tokens that stay visible before a window, kSinks has those, kNorm a norm and those, if there are any.  With first
// tokens blocks count on without a gap: first theirs, then the window's, from v0 on; block_of() says which block of the sequence that is.
enum Kind { kPlain, kSinks, kNorm };
template <int D, Kind KIND>
__global__ __launch_bounds__(WAVES * 64, D > 128 ? 1 : D > 64 ? 3 : 4) void kv_rows_kernel(KvAttentionParams p) {
    constexpr bool SINKS = KIND != kPlain, NORM = KIND == kNorm;
    constexpr int C = D / 32;                    // runs of 32 channels = steps of K Q^T per 16 tokens
    constexpr int kRow = row_floats(D);
    extern __shared__ __attribute__((aligned(16))) float lds[];
    const int cap = p.row_cap;                   // rows that a tile can have
    float *sums = lds, *ml = lds + WAVES * cap * kRow;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, q4 = lane >> 4;
    const int head = blockIdx.y, b = blockIdx.z / p.row_tiles, tile = blockIdx.z % p.row_tiles;
    int t0, n;
    kv_range(p.batch.cu, b, p.batch.total, t0, n);
    const int len = __builtin_amdgcn_readfirstlane(kv_length(p.cache, p.batch, p.batch.kv_len[b])), rows = n * p.group;
    if (tile * 16 >= rows || rows > p.most_rows) return;
    // the lane's row and the keys [seen_lo, seen_hi) that it sees
    const int r = tile * 16 + l16 < rows ? tile * 16 + l16 : rows - 1;
    const int tok = r / p.group, qh = head * p.group + r % p.group, pos = len - n + tok;
    const auto hi_of = [&](int at) { return at < 0 ? 0 : p.causal ? at + 1 : len; };      // (a token without a position sees nothing)
    const int seen_hi = hi_of(pos);
    const int seen_lo = p.causal && p.window > 0 && pos + 1 > p.window ? pos + 1 - p.window : 0;
    // keys of the row between the first tokens and its window
    const int hidden = SINKS && p.sinks < seen_lo ? p.sinks : seen_lo;
    const uint32_t hidden_count = (uint32_t)(seen_lo - hidden);
    // of the tile: its first row sees the fewest and the earliest keys
    const int tok_a = tile * 16 / p.group, last = tile * 16 + 15 < rows ? tile * 16 + 15 : rows - 1, tok_z = last / p.group;
    const int pos_a = len - n + tok_a, pos_z = len - n + tok_z;
    const int any_hi = hi_of(pos_z), all_hi = hi_of(pos_a);
    const int any_lo = p.causal && p.window > 0 && pos_a + 1 > p.window ? pos_a + 1 - p.window : 0, all_lo = p.causal && p.window > 0 && pos_z + 1 > p.window ? pos_z + 1 - p.window : 0;
    const int blk0 = any_lo >> 5, blk1 = (any_hi + 31) >> 5;
    const int sinks = SINKS ? p.sinks : 0, sink_blocks = (int)(((long long)sinks + 31) >> 5), v0 = SINKS ? blk0 - (sink_blocks < blk0 ? sink_blocks : blk0) : blk0;
    const auto block_of = [&](int v) { return SINKS && v < blk0 ? v - v0 : v; };
    // this workgroup's blocks
    const int chunk = blockIdx.x, count = blk1 > blk0 ? blk1 - v0 : 0;
    int nchunks = (count + p.chunk_blocks - 1) / p.chunk_blocks;
    nchunks = nchunks < 1 ? 1 : nchunks > p.chunks ? p.chunks : nchunks;
    if (chunk >= nchunks) return;
    const int c0 = v0 + chunk * p.chunk_blocks, c1 = chunk == nchunks - 1 ? blk1 : c0 + p.chunk_blocks;

    const int32_t *table = p.batch.table + (size_t)b * p.batch.table_width;
    const int bs = p.cache.page_shift - 5;
    // The wavefront's blocks c0 + wave + WAVES i: their pages and scale bytes, 64 blocks at a time, one in a lane
    int base = c0 + wave, left = base < c1 ? (c1 - base + WAVES - 1) / WAVES : 0, here = 0, page_l = -1, kb_l = 0, vb_l = 0;
    auto look_up = [&]() {
        here = left < 64 ? left : 64;
        page_l = here == 0 ? -1 : table[block_of(base + WAVES * (lane < here ? lane : 0)) >> bs];
    };
    auto look_up_bytes = [&]() {
        const int blk = block_of(base + WAVES * lane);
        const bool named = lane < here && (uint32_t)page_l < (uint32_t)p.cache.pages;
        const size_t u = named ? (((size_t)page_l * p.cache.heads + head) << bs) + (blk & ((1 << bs) - 1)) : 0;
        page_l = named ? page_l : -1;
        kb_l = p.cache.ks[u];
        vb_l = p.cache.vs[u];
    };
    const uint32_t k_off = (uint32_t)((16 * (l16 >> 3) + (l16 & 7)) * D + 16 * q4), v_off = (uint32_t)((l16 * 4 + q4) * 16);
    // Block i of the wavefront.  Past the last one, or where the table names no page, every lane reads the first 16 bytes of the cache: loads are issued
    // whether they are needed or not, so that a wait for one block leaves the next ones in flight.
    auto load = [&](Block<D> &t, int i) {
        const int page = __builtin_amdgcn_readlane(page_l, i < here ? i : 0);
        const bool real = i < here && page >= 0;
        const size_t u = real ? (((size_t)page * p.cache.heads + head) << bs) + (block_of(base + WAVES * i) & ((1 << bs) - 1)) : 0;
        const uint8_t *k = p.cache.k + u * (32 * D), *v = p.cache.v + u * (32 * D);
        const uint32_t ko = real ? k_off : 0u, vo = real ? v_off : 0u;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int c = 0; c < D / 64; ++c) t.k[j][c] = *reinterpret_cast<const uint4 *>(k + ko + 8 * j * D + 64 * c);
#pragma unroll
        for (int a = 0; a < D / 32; ++a) t.v[a] = *reinterpret_cast<const uint4 *>(v + vo + 1024 * a);
    };
    look_up();
    // The queries, a step of the wavefronts each: requested before the blocks, whose addresses wait for the table
    constexpr int kMine = (C + WAVES - 1) / WAVES;      // steps of a wavefront (D = 64: of the first two)
    const auto place = [&](int i) {                     // step c: channels 64 (c / 2) + 16 q4 + 8 (c % 2) .. + 7
        const int c = wave * kMine + i < C ? wave * kMine + i : C - 1;
        return 64 * (c / 2) + 16 * q4 + 8 * (c % 2);
    };
    std::conditional_t<NORM, KvReadying<kMine>, KvRotating<kMine>> turning;
    const uint16_t *row = p.q.data + (size_t)(t0 + tok) * p.q.token_stride + qh * p.q.head_stride;
    if constexpr (NORM) turning.request(row, p.norm, p.rope, pos, qh, place, p.cache.k);
    else turning.request(row, p.rope, pos, place);
    __builtin_amdgcn_sched_barrier(0);
    look_up_bytes();
    Block<D> even, odd;
    load(even, 0);
    load(odd, 1);
    __builtin_amdgcn_sched_barrier(0);
    // f16 of the rotated row times a power of two that brings its largest element to [2^14, 2^15)
    kv_f16x8 qf[C];
    float to_t;      // score -> exponent of 2, but for the block's scale
    {
        float x[kMine][8];
        turning.finish(p.rope, place, x);
        uint32_t top = 0u;
        float sum = 0.f, tiny = 0.f;
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t u = __float_as_uint(x[i][e]) & 0x7fffffffu;
                top = top > u ? top : u;
            }
            if (wave * kMine + i < C) {
                if constexpr (NORM) turning.add_squares(i, sum, tiny);
                float *dst = lds + ((wave * kMine + i) * 64 + lane) * 8;
                *reinterpret_cast<kv_floatx4 *>(dst) = kv_floatx4{x[i][0], x[i][1], x[i][2], x[i][3]};
                *reinterpret_cast<kv_floatx4 *>(dst + 4) = kv_floatx4{x[i][4], x[i][5], x[i][6], x[i][7]};
            }
        }
        lds[C * 512 + wave * 64 + lane] = kv_max32(kv_max16(__uint_as_float(top >= 0x7f800000u ? 0x7f800000u : top)));
        if (NORM) {
            lds[C * 512 + (WAVES + wave) * 64 + lane] = kv_sum32(kv_sum16(sum));
            lds[C * 512 + (2 * WAVES + wave) * 64 + lane] = kv_sum32(kv_sum16(tiny));
        }
        kv_lds_barrier();
        float m = lds[C * 512 + lane];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) m = fmaxf(m, lds[C * 512 + w * 64 + lane]);
        float factor = 1.f;
        if (NORM) {
            float squares[2] = {0.f, 0.f};
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                squares[0] += lds[C * 512 + (WAVES + w) * 64 + lane];
                squares[1] += lds[C * 512 + (2 * WAVES + w) * 64 + lane];
            }
            const bool large = kv_norm_leaves(squares[0], 1.f / D, p.norm.eps);
            factor = kv_norm_factor(large ? squares[1] : squares[0], 1.f / D, kv_norm_eps(large, p.norm.eps)) * (large ? kKvTiny / kHeld : 1.f / kHeld);
        }
        const int e = (int)(__float_as_uint(m) >> 23) - 127;                          // m in [2^e, 2^(e + 1))
        const int up = e < -100 ? 114 : e > 127 ? 0 : 14 - e;                         // (not finite: as it is, the row becomes NaN)
        const float f = kv_pow2(up);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const kv_floatx4 lo = *reinterpret_cast<const kv_floatx4 *>(lds + (c * 64 + lane) * 8), hi = *reinterpret_cast<const kv_floatx4 *>(lds + (c * 64 + lane) * 8 + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                qf[c][i] = (_Float16)(lo[i] * f);
                qf[c][4 + i] = (_Float16)(hi[i] * f);
            }
        }
        to_t = p.scale * kv_pow2(-up) * factor;
    }

    kv_floatx4 o[D / 16] = {};
    float m = kNone, l = 0.f;
    int ref = 0;                                 // byte of the reference scale of the values in o

    // exponents t of block i's weights, -inf where the row does not see the token; values of tokens that do not exist are cleared
    auto scores = [&](Block<D> &cur, int i, float (&t)[8]) {
        const int v = base + WAVES * i, blk = block_of(v), kb = __builtin_amdgcn_readlane(kb_l, i);
        const bool named = __builtin_amdgcn_readlane(page_l, i) >= 0;
        kv_floatx4 s[2] = {};
#pragma unroll
        for (int c = 0; c < D / 64; ++c)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                s[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kv_f16_of(cur.k[j][c].x, cur.k[j][c].y, 1.f), qf[2 * c], s[j], 0, 0, 0);
                s[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kv_f16_of(cur.k[j][c].z, cur.k[j][c].w, 1.f), qf[2 * c + 1], s[j], 0, 0, 0);
            }
        // the lane's eight tokens are those of slot q4
        const float f = kv_within_range(to_t * kv_pow2(kb - 127));      // (a sum of zero times it is zero)
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] = s[j / 4][j % 4] * f;
        if (!named || v * kKvBlock < all_lo || v * kKvBlock + kKvBlock > all_hi) {      // (before the window: less than all_lo)
            const int first = blk * kKvBlock + kv_slot_token(q4);
            uint32_t live[2] = {~0u, ~0u};       // bytes of the codes of tokens that exist
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int key = first + (j & 3) + 8 * (j >> 2);
                const bool ok = named && (SINKS ? (uint32_t)(key - hidden) >= hidden_count : key >= seen_lo) && key < seen_hi && key < len;
                t[j] = ok ? t[j] : -__builtin_inff();
                if (!named || key >= len) live[j >> 2] &= ~(0xffu << (8 * (j & 3)));
            }
#pragma unroll
            for (int a = 0; a < D / 32; ++a) {
                cur.v[a].x &= live[0]; cur.v[a].y &= live[1]; cur.v[a].z &= live[0]; cur.v[a].w &= live[1];
            }
        }
    };
    auto largest_of = [&](const float (&t)[8]) {      // of the row
        float top = t[0];
#pragma unroll
        for (int j = 1; j < 8; ++j) top = fmaxf(top, t[j]);
        return kv_max32(kv_max16(top));
    };
    auto weights = [&](const float (&t)[8], float from, float &sum) {      // and the sum of what is multiplied
        kv_f16x8 pf;
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            const kv_f16x2 e = {(_Float16)__builtin_amdgcn_exp2f(t[j] - from + kShift), (_Float16)__builtin_amdgcn_exp2f(t[j + 1] - from + kShift)};
            sum = __builtin_amdgcn_fdot2(e, kv_f16x2{(_Float16)1.f, (_Float16)1.f}, sum, false);
            pf[j] = e[0];
            pf[j + 1] = e[1];
        }
        return pf;
    };
    auto step = [&](Block<D> &cur, int i) {
        const int vb = __builtin_amdgcn_readlane(vb_l, i);
        float t[8];
        scores(cur, i, t);
        const float top = largest_of(t);
        const int ref_new = vb > ref ? vb : ref;
        if (__builtin_amdgcn_ballot_w64(top > m + kSlack) != 0ull || ref_new != ref) {
            const float m_new = fmaxf(m, top), keep = __builtin_amdgcn_exp2f(m - m_new);
            l *= keep;
            const float both = keep * kv_pow2(ref - ref_new);
#pragma unroll
            for (int d = 0; d < D / 16; ++d) o[d] *= both;
            m = m_new;
            ref = ref_new;
        }
        const kv_f16x8 pf = weights(t, m, l);
        const float vf = kv_pow2(vb - ref);
#pragma unroll
        for (int a = 0; a < D / 32; ++a) {
            o[2 * a] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kv_f16_of(cur.v[a].x, cur.v[a].y, vf), pf, o[2 * a], 0, 0, 0);
            o[2 * a + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kv_f16_of(cur.v[a].z, cur.v[a].w, vf), pf, o[2 * a + 1], 0, 0, 0);
        }
    };
    KvSpread spread;
    bool wide = false;      // the values' scales are too far apart for one reference
    for (;;) {
        wide = spread.add(page_l >= 0 ? vb_l : 0);
        if (wide) break;
        for (int i = 0; i < here; i += 2) {
            step(even, i);
            load(even, i + 2);
            __builtin_amdgcn_sched_barrier(0);
            if (i + 1 < here) step(odd, i + 1);
            load(odd, i + 3);
            __builtin_amdgcn_sched_barrier(0);
        }
        left -= here;
        if (left <= 0) break;
        base += WAVES * 64;
        look_up();
        look_up_bytes();
        load(even, 0);
        load(odd, 1);
    }
    int row_ref = ref;
    if (__builtin_expect(wide, 0)) {      // from the start, a block at a time
#pragma unroll
        for (int d = 0; d < D / 16; ++d) o[d] = kv_floatx4{};
        m = kNone;
        l = 0.f;
        row_ref = 0;
        base = c0 + wave;
        left = (c1 - base + WAVES - 1) / WAVES;
        for (;;) {
            look_up();
            look_up_bytes();
            for (int i = 0; i < here; ++i) {
                load(even, i);
                float t[8];
                scores(even, i, t);
                const float top = largest_of(t);
                float sum = 0.f, largest = 0.f;
                const kv_f16x8 pf = weights(t, top > -__builtin_inff() ? top : 0.f, sum);
#pragma unroll
                for (int d = 0; d < D / 16; ++d)
#pragma unroll
                    for (int j = 0; j < 4; ++j) largest = fmaxf(largest, __builtin_fabsf(o[d][j]));
                const KvJoin join = kv_join(m, row_ref, top, __builtin_amdgcn_readlane(vb_l, i), kv_max32(kv_max16(largest)));
                l = l * join.keep_l + sum * join.add_l;
#pragma unroll
                for (int a = 0; a < D / 32; ++a) {
                    const kv_floatx4 x = __builtin_amdgcn_mfma_f32_16x16x32_f16(kv_f16_of(even.v[a].x, even.v[a].y, 1.f), pf, kv_floatx4{}, 0, 0, 0);
                    const kv_floatx4 y = __builtin_amdgcn_mfma_f32_16x16x32_f16(kv_f16_of(even.v[a].z, even.v[a].w, 1.f), pf, kv_floatx4{}, 0, 0, 0);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        o[2 * a][j] = __builtin_amdgcn_ldexpf(o[2 * a][j] * join.keep, join.keep_e) + __builtin_amdgcn_ldexpf(x[j] * join.add, join.add_e);
                        o[2 * a + 1][j] = __builtin_amdgcn_ldexpf(o[2 * a + 1][j] * join.keep, join.keep_e) + __builtin_amdgcn_ldexpf(y[j] * join.add, join.add_e);
                    }
                }
            }
            left -= here;
            if (left <= 0) break;
            base += WAVES * 64;
        }
    }

    // ---- the wavefronts meet: as weighted means of values, which pass no range that the values themselves keep (their sums may) ----
    __syncthreads();      // (the queries lay there)
    l = kv_sum32(kv_sum16(l));
    if (q4 == 0) {
        ml[(wave * 16 + l16) * 2] = m;
        ml[(wave * 16 + l16) * 2 + 1] = l;
    }
    if (l16 < cap) {
        const float inv = kv_inverse(l);
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
            kv_floatx4 x;
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = __builtin_amdgcn_ldexpf(o[d][j] * inv, row_ref - 127);
            *reinterpret_cast<kv_floatx4 *>(sums + (wave * cap + l16) * kRow + 16 * d + 4 * q4) = x;
        }
    }
    __syncthreads();
    // pieces of four channels of a row
    const long long part = ((long long)blockIdx.z * p.cache.heads + head) * p.chunks;      // of this row tile's parts
    const int live_rows = rows - tile * 16 < cap ? rows - tile * 16 : cap, pieces = live_rows * (D / 4);      // (tokens past max_new have no room, and no row)
    const size_t part_floats = (size_t)cap * (D + 2);      // [cap][D] weighted means, [cap][2] maximum and sum of weights
    const __amdgpu_buffer_rsrc_t rs = make_rsrc(p.partial + part * part_floats, (size_t)nchunks * part_floats * 4);
    auto store = [&](int row, int d, kv_floatx4 x) {
        const int rr = tile * 16 + row;
        uint16_t *dst = p.out + ((size_t)(t0 + rr / p.group) * p.q_heads + head * p.group + rr % p.group) * D + d;
        const kv_bf16x2 lo = {(__bf16)x[0], (__bf16)x[1]}, hi = {(__bf16)x[2], (__bf16)x[3]};
        *reinterpret_cast<uint2 *>(dst) = make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
    };
    for (int i = threadIdx.x; i < pieces; i += WAVES * 64) {
        const int row = i / (D / 4), d = i % (D / 4) * 4;
        float top = kNone;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) top = fmaxf(top, ml[(w * 16 + row) * 2]);
        float weight[WAVES], sum = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            weight[w] = ml[(w * 16 + row) * 2 + 1] * __builtin_amdgcn_exp2f(ml[(w * 16 + row) * 2] - top);
            sum += weight[w];
        }
        const float inv = kv_inverse(sum);
        kv_floatx4 x = {};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) x += *reinterpret_cast<const kv_floatx4 *>(sums + (w * cap + row) * kRow + d) * (weight[w] * inv);
        if (nchunks > 1) {      // past the L2 of this XCD: the workgroup that adds the parts may run on another
            const int at = (int)(chunk * part_floats * 4);
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(kv_u32x4, x), rs, at + (row * D + d) * 4, 0, kAgent);
            if (d == 0) __builtin_amdgcn_raw_buffer_store_b64(kv_u32x2{__float_as_uint(top), __float_as_uint(sum)}, rs, at + (cap * D + row * 2) * 4, 0, kAgent);
        } else {
            store(row, d, x);
        }
    }
    if (nchunks == 1) return;

    // ---- the parts of the row tile meet: the arrival words hold anything but kKvArrived until a workgroup marks its own, and are cleared at the end ----
    __shared__ int missing;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // this wavefront's stores are acknowledged
    if (threadIdx.x == 0) missing = 0;
    __syncthreads();
    unsigned long long *words = p.arrived + part;
    if (wave == 0) {
        if (lane == 0) (void)__hip_atomic_exchange(words + chunk, kKvArrived, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        bool all = true;
        for (int i = lane; i < nchunks; i += 64) all = all && __hip_atomic_load(words + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == kKvArrived;
        if (__builtin_amdgcn_ballot_w64(!all) != 0ull && lane == 0) missing = 1;
    }
    __syncthreads();
    if (missing) return;
    // weights of the parts, [chunk][row], of sum 1 in a row; thread groups add every so many parts, and the groups meet in LDS
    float *weight = lds, *meet = lds + ((nchunks * cap + 3) & ~3);
    for (int row = wave; row < live_rows; row += WAVES) {
        float mx = kNone, part_m[kKvMostChunks / 64], part_l[kKvMostChunks / 64];
#pragma unroll
        for (int k = 0; k < kKvMostChunks / 64; ++k) {
            const int c = lane + 64 * k;
            kv_u32x2 w = {__float_as_uint(kNone), 0u};
            if (c < nchunks) w = __builtin_amdgcn_raw_buffer_load_b64(rs, (int)((c * part_floats + cap * D + row * 2) * 4), 0, kAgent);
            part_m[k] = __uint_as_float(w[0]);
            part_l[k] = __uint_as_float(w[1]);
            mx = fmaxf(mx, part_m[k]);
        }
#pragma unroll
        for (int s = 1; s < 64; s *= 2) mx = fmaxf(mx, __shfl_xor(mx, s));
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < kKvMostChunks / 64; ++k) {
            part_l[k] *= __builtin_amdgcn_exp2f(part_m[k] - mx);
            sum += part_l[k];
        }
#pragma unroll
        for (int s = 1; s < 64; s *= 2) sum += __shfl_xor(sum, s);
        const float inv = kv_inverse(sum);
#pragma unroll
        for (int k = 0; k < kKvMostChunks / 64; ++k)
            if (lane + 64 * k < nchunks) weight[(lane + 64 * k) * cap + row] = part_l[k] * inv;
    }
    __syncthreads();
    const int groups = pieces < WAVES * 64 ? WAVES * 64 / pieces : 1, mine = threadIdx.x / pieces;
    for (int i0 = 0; i0 < pieces; i0 += WAVES * 64) {      // (more than one round: one group)
        const int i = groups > 1 ? threadIdx.x % pieces : i0 + threadIdx.x, row = i / (D / 4), d = i % (D / 4) * 4;
        const bool works = groups > 1 ? mine < groups : i < pieces;
        kv_floatx4 x = {};
        if (works) {
            const int first = groups > 1 ? mine : 0;
            constexpr int kAhead = 8;
            for (int c0 = first; c0 < nchunks; c0 += kAhead * groups) {
                kv_floatx4 y[kAhead];
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    const int c = c0 + k * groups < nchunks ? c0 + k * groups : c0;
                    y[k] = __builtin_bit_cast(kv_floatx4, __builtin_amdgcn_raw_buffer_load_b128(rs, (int)((c * part_floats + row * D + d) * 4), 0, kAgent));
                }
#pragma unroll
                for (int k = 0; k < kAhead; ++k)
                    if (c0 + k * groups < nchunks) x += y[k] * weight[(c0 + k * groups) * cap + row];
            }
        }
        if (groups > 1) {
            if (works) *reinterpret_cast<kv_floatx4 *>(meet + threadIdx.x * 4) = x;
            __syncthreads();
            if (mine == 0) {
                for (int g = 1; g < groups; ++g) x += *reinterpret_cast<const kv_floatx4 *>(meet + (g * pieces + threadIdx.x) * 4);
                store(row, d, x);
            }
        } else if (works) {
            store(row, d, x);
        }
    }
    // (every workgroup of the row tile has made its mark; two that both found all marks store the same results)
    for (int i = threadIdx.x; i < nchunks; i += WAVES * 64) __hip_atomic_store(words + i, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

template <int D, Kind KIND>
hipError_t launch_rows_of(const KvAttentionParams &p, hipStream_t stream) {
    static LdsLimit limit;
    constexpr int most = rows_lds_bytes(D, WAVES, 16, kKvMostChunks, KIND == kNorm);
    if (p.chunks > kKvMostChunks) return hipErrorInvalidValue;
    if (most > 65536) {
        const hipError_t e = limit.raise(reinterpret_cast<const void *>(kv_rows_kernel<D, KIND>), most);
        if (e != hipSuccess) return e;
    }
    kv_rows_kernel<D, KIND><<<dim3(p.chunks, p.cache.heads, p.batch.sequences * p.row_tiles), WAVES * 64, rows_lds_bytes(D, WAVES, p.row_cap, p.chunks, KIND == kNorm), stream>>>(p);
    return hipGetLastError();
}

template <int D>
hipError_t launch_rows(const KvAttentionParams &p, hipStream_t stream) {
    return p.norm.on ? launch_rows_of<D, kNorm>(p, stream) : p.sinks > 0 ? launch_rows_of<D, kSinks>(p, stream) : launch_rows_of<D, kPlain>(p, stream);
}

}  // namespace

hipError_t launch_kv_attention_rows(const KvAttentionParams &p, hipStream_t stream) {
    switch (p.cache.dim) {
        case 64: return launch_rows<64>(p, stream);
        case 128: return launch_rows<128>(p, stream);
        case 256: return launch_rows<256>(p, stream);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace svdq
