// Compaction of the paged 8-bit cache (layout: kv_common.h): tokens of a sequence move to other places, and the blocks there are quantized anew.
//
//   token first + i of a sequence becomes what its token f_i was:  k' = R(first + i) R(f_i)^-1 k (k' = k without a rotation, and where a token keeps its position),  v' = v
//
// Where a pair of channels was turned by (c0, s0) and is to be turned by (c1, s1), it is turned by ((c1 c0 + s1 s0) / m, (s1 c0 - c1 s0) / m), m = c0^2 + s0^2, in fp32: tables
// that scale their cosines and sines keep that scale.  Blocks are written as an append of the moved vectors would: byte of the smallest power of two, codes rounded once, the larger
// byte where a block holds tokens already.  A vector with an element that is not finite, or of a token that no page of the sequence holds, is NaN codes and zeros.
//
// Work split: a workgroup of four wavefronts has one block of the new place and one or more heads in turn, two wavefronts the keys and two the values.  A token's key is a row of
// codes and is read as it lies.  Its values are single bytes, 64 to a token and run of 32 channels, spread over the whole block of the old place: the old
// blocks go through LDS, four at a time, rows of 64 bytes laid 80 apart so that 16 rows and 4 slots lie on 64 banks, and are picked there byte by byte.
// Moves within the same pages go by way of the workspace: every block is made there first, a second kernel puts them in place, and their order does not matter.
// Of values every line of an old block holds all of its tokens, so blocks are read whole, and twice where neighbouring new blocks share one.  The rows of the next head are in flight
// while this one's are picked and written.
// Bound: memory.  64 sequences of 9000 to 16384 tokens, eight heads of 128, of which 5000 to 12001 stay, keys turned: 622 us, in which 3.4 GB pass the L2s (2.32 read,
// 1.11 written), 5.5 TB/s; the plain reading back of the same rows moves 3.35 GB at 5.0.  It is more than it needs: the keys that stay and old blocks of values, whole and once, are 1.36 GB; the rotation's
// rows, two a token, are 0.48, and the rest are old blocks that two new ones share (without turning 595 us, 2.95 GB; where the latest stay, 567 and 2.7).  At 128 registers four workgroups stay on a CU (three, at 131: 780 us; five spill).
// 16 sequences with lists for each head, two fifths kept: 76 us, 267 MB (183 read), 3.5 TB/s, a chain of tokens, pages, blocks and their picking for each head, eleven rounds of workgroups (two to four heads a
// workgroup 75 to 79).  A few tokens of 32 sequences: 7.8 us, and 4.0 to put them in place.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.h"
#include "kv_blocks.h"
#include "kv_common.h"

namespace svdq {
namespace {

constexpr int kStages = 4;          // old blocks in LDS at a time
constexpr int kStageRow = 80;       // bytes apart of rows of 64
template <int D> constexpr int kStageBytes = D / 32 * 16 * kStageRow;

template <int D> struct Shelf {      // the old blocks of values in LDS, and how a token is found there
    __attribute__((aligned(16))) unsigned char blocks[kStages * kStageBytes<D>];
    uint32_t spot[kKvBlock];
    float scale[kKvBlock];
};

struct Place { BlockWork w; int sequence; };
// The new place's block of a work item; w.lo >= w.hi: none.  row0: the move that its token 0 would be.
__device__ __forceinline__ Place place_of(const KvCompactParams &p, int number) {
    const long long cap = (long long)p.batch.table_width << p.to.page_shift;
    const auto first_of = [&](int value) { return value < 0 ? 0 : (long long)value > cap ? (int)cap : value; };
    const auto end_of = [&](int first, int n) { return (long long)first + n > cap ? (int)cap : first + n; };
    const KvItem item = kv_item(p.batch, number, [&](int n, int value) {
        const int first = first_of(value), end = end_of(first, n);
        return end > first ? ((end + 31) >> 5) - (first >> 5) : 0;
    });
    const int first = first_of(item.value), end = end_of(first, item.count);
    Place at;
    at.sequence = item.sequence;
    at.w.blk = (first >> 5) + item.local;
    at.w.lo = first > at.w.blk * kKvBlock ? first - at.w.blk * kKvBlock : 0;
    at.w.hi = item.local < 0 || item.count == 0 ? 0 : end - at.w.blk * kKvBlock < kKvBlock ? end - at.w.blk * kKvBlock : kKvBlock;
    at.w.row0 = (long long)item.first + (at.w.blk * kKvBlock - first);
    return at;
}

// Where the tokens of a block come from, token `lane % 32` in a lane.
struct Sources {
    uint32_t unit;      // block of the old place, as an index of the scale arrays, of head 0; ~0: no such token
    int token;          // old position
    __device__ __forceinline__ void find(const KvCompactParams &p, const Place &at, int h, int lane) {
        const long long move = at.w.row0 + readable(at.w, lane & 31);
        token = p.from_token[(p.per_head ? (size_t)h * p.batch.total : 0) + move];
        const int bs = p.from.page_shift - 5;
        const bool within = (uint32_t)token < (uint32_t)p.from_width << p.from.page_shift;
        const int page = within ? p.from_table[(size_t)at.sequence * p.from_width + (token >> p.from.page_shift)] : -1;
        unit = (uint32_t)page < (uint32_t)p.from.pages ? (((uint32_t)page * (uint32_t)p.from.heads) << bs) + (uint32_t)((token >> 5) & ((1 << bs) - 1)) : ~0u;
    }
    __device__ __forceinline__ size_t of_head(const KvCompactParams &p, int h) const { return unit == ~0u ? 0 : (size_t)unit + ((size_t)h << (p.from.page_shift - 5)); }
    // Runs of tokens out of one old block: in which run the lane's token is, and how many there are
    __device__ __forceinline__ int runs(int lane, int &mine, unsigned long long &starts) const {
        const uint32_t before = (uint32_t)__shfl((int)unit, lane == 0 ? 0 : lane - 1);
        starts = __builtin_amdgcn_ballot_w64((lane & 31) == 0 || unit != before) & 0xffffffffull;
        mine = __builtin_popcountll(starts & ((2ull << (lane & 31)) - 1ull)) - 1;
        return __builtin_popcountll(starts);
    }
};
__device__ __forceinline__ float code_number(uint32_t code, float scale) { return __builtin_amdgcn_cvt_scalef32_f32_fp8(code, scale, 0); }
__device__ __forceinline__ void code_numbers(uint2 w, float scale, float (&x)[8]) {
    const kv_floatx2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w.x, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w.x, scale, true);
    const kv_floatx2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w.y, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w.y, scale, true);
    x[0] = a[0]; x[1] = a[1]; x[2] = b[0]; x[3] = b[1]; x[4] = c[0]; x[5] = c[1]; x[6] = d[0]; x[7] = d[1];
}
__device__ __forceinline__ float byte_scale(int byte) { return kv_pow2((byte < 1 ? 1 : byte) - 127); }      // (byte 0: the codes are zeros)

// Where a head's block goes, and where the tokens that it holds already lie.
struct Target { uint8_t *codes, *byte; const uint8_t *old; };

// The keys of half a block, 16 tokens: units of 16 channels, the two runs of eight that the rotation pairs (as in the append).
template <int D>
struct KeyMoves {
    static constexpr int U = D / 16, N = U / 4;
    const KvCompactParams &p;
    const Place &at;
    const int lane, half;
    int chan[2];
    uint2 raw[N][2];
    int byte[N];
    float c[N][8], s[N][8], x[N][2][8], top[N];
    bool stays[N];      // at its position
    __device__ __forceinline__ int token(int i) const { return 16 * half + (lane + 64 * i) / U; }
    __device__ __forceinline__ KeyMoves(const KvCompactParams &p_, const Place &at_, int lane_, int half_) : p(p_), at(at_), lane(lane_), half(half_) {
        const int pr = lane % U;
        const bool halves = !p.rope.interleaved && pr < p.rope.dims / 16;
        chan[0] = halves ? pr * 8 : pr * 16;
        chan[1] = halves ? pr * 8 + p.rope.dims / 2 : pr * 16 + 8;
    }
    __device__ __forceinline__ void load(const Sources &src, int h) {
        const size_t unit = src.of_head(p, h);
        const int byte_l = p.from.ks[unit];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t u0 = (uint32_t)__shfl((int)src.unit, token(i));
            const int t = __shfl(src.token, token(i));
            const size_t u = u0 == ~0u ? 0 : (size_t)u0 + ((size_t)h << (p.from.page_shift - 5));
            const uint8_t *row = p.from.k + u * (32 * D) + (u0 == ~0u ? 0 : t & 31) * D;
            raw[i][0] = *reinterpret_cast<const uint2 *>(row + chan[0]);
            raw[i][1] = *reinterpret_cast<const uint2 *>(row + chan[1]);
            byte[i] = __shfl(byte_l, token(i));
            if (u0 == ~0u) raw[i][0].x = raw[i][0].y = raw[i][1].x = raw[i][1].y = kKvNaN * 0x01010101u;
        }
    }
    __device__ __forceinline__ void angles(const Sources &src) {
        if (p.rope.dims == 0) return;
        const int half_dims = p.rope.dims / 2;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int last = p.rope.dims / 16 - 1, pr = lane % U, to = at.w.blk * kKvBlock + readable(at.w, token(i)), from = __shfl(src.token, token(i));
            const auto row = [&](int pos) { return p.rope.table + (size_t)(pos < 0 ? 0 : pos < p.rope.positions ? pos : p.rope.positions - 1) * p.rope.dims + (pr < last ? pr : last) * 8; };
            float c0[8], s0[8], c1[8], s1[8];
            kv_load8(row(from), c0);
            kv_load8(row(from) + half_dims, s0);
            kv_load8(row(to), c1);
            kv_load8(row(to) + half_dims, s1);
            stays[i] = from == to;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float size = __builtin_fmaf(c0[e], c0[e], s0[e] * s0[e]), near = __builtin_amdgcn_rcpf(size);
                const float m = __builtin_fmaf(__builtin_fmaf(-size, near, 1.f), near, near);      // 1 / size, a step of Newton's on the instruction's
                c[i][e] = __builtin_fmaf(c1[e], c0[e], s1[e] * s0[e]) * m;
                s[i][e] = __builtin_fmaf(s1[e], c0[e], -(c1[e] * s0[e])) * m;
            }
        }
    }
    __device__ __forceinline__ void gather(const Sources &, int, int, Shelf<D> &, int runs) {
        for (int done = 0; done < runs; done += kStages) {      // (the values' wavefronts do)
            if (done > 0) kv_lds_barrier();
            kv_lds_barrier();
        }
    }
    // turns the rows; returns the tokens with an element that is not finite.  Asks for the rows of head `next`, if there is one
    __device__ __forceinline__ uint32_t look(const Sources &src, int next) {
        uint32_t bad = 0u;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float scale = byte_scale(byte[i]);
            code_numbers(raw[i][0], scale, x[i][0]);
            code_numbers(raw[i][1], scale, x[i][1]);
        }
        if (next >= 0) load(src, next);      // (its rows are in flight while this head's are worked on)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (lane % U < p.rope.dims / 16 && !stays[i]) {
                if (p.rope.interleaved) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float a = x[i][e / 4][2 * (e % 4)], y = x[i][e / 4][2 * (e % 4) + 1];
                        x[i][e / 4][2 * (e % 4)] = kv_turn_fma_a(a, y, c[i][e], s[i][e]);
                        x[i][e / 4][2 * (e % 4) + 1] = kv_turn_fma_b(a, y, c[i][e], s[i][e]);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float a = x[i][0][e], y = x[i][1][e];
                        x[i][0][e] = kv_turn_fma_a(a, y, c[i][e], s[i][e]);
                        x[i][1][e] = kv_turn_fma_b(a, y, c[i][e], s[i][e]);
                    }
                }
            }
            float m = 0.f;      // (NaN if one is NaN)
#pragma unroll
            for (int e = 0; e < 8; ++e) m = __builtin_elementwise_maximum(__builtin_elementwise_maximum(m, __builtin_fabsf(x[i][0][e])), __builtin_fabsf(x[i][1][e]));
            top[i] = live(at.w, token(i)) ? m : 0.f;
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
    __device__ __forceinline__ void write(const Target &to, const BlockScale &sc, uint32_t bad) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int place = token(i) * D;
            if (token(i) < at.w.lo && (sc.grown || to.old != to.codes)) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint2 v = *reinterpret_cast<const uint2 *>(to.old + place + chan[j]);
                    *reinterpret_cast<uint2 *>(to.codes + place + chan[j]) = sc.grown ? make_uint2(kv_rescale4(v.x, sc.old_factor), kv_rescale4(v.y, sc.old_factor)) : v;
                }
            }
            if (!live(at.w, token(i))) continue;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float (&y)[8] = x[i][j];
                uint2 v = make_uint2(codes4(y[0], y[1], y[2], y[3], sc.scale), codes4(y[4], y[5], y[6], y[7], sc.scale));
                if (bad != 0u && (bad >> token(i)) & 1u) v.x = v.y = kKvNaN * 0x01010101u;
                *reinterpret_cast<uint2 *>(to.codes + place + chan[j]) = v;
            }
        }
    }
};

// The values of a block, D / 64 pieces of 16 bytes a lane: the two channels of a place for the eight tokens of slot lane % 4.
template <int D>
struct ValueMoves {
    static constexpr int N = D / 64;
    const KvCompactParams &p;
    const Place &at;
    const int lane, half;
    kv_u32x4 staged[kStages][N];
    float x[N][2][8], top[8];
    int byte_l;                  // of the lane's token
    __device__ __forceinline__ int token(int j) const { return kv_slot_token(lane & 3) + (j & 3) + 8 * (j >> 2); }
    __device__ __forceinline__ int piece(int i) const { return lane + 64 * half + 128 * i; }
    __device__ __forceinline__ ValueMoves(const KvCompactParams &p_, const Place &at_, int lane_, int half_) : p(p_), at(at_), lane(lane_), half(half_) {}
    __device__ __forceinline__ void load_runs(const Sources &src, int h, int first, unsigned long long starts) {      // up to kStages of them, from the first-th on
        for (int n = 0; n < first; ++n) starts &= starts - 1;
        size_t unit[kStages];
        bool some[kStages];
#pragma unroll
        for (int k = 0; k < kStages; ++k) {
            some[k] = starts != 0ull;
            const uint32_t u0 = (uint32_t)__builtin_amdgcn_readlane((int)src.unit, some[k] ? __builtin_ctzll(starts) : 0);
            unit[k] = u0 == ~0u ? 0 : (size_t)u0 + ((size_t)h << (p.from.page_shift - 5));
            starts &= starts - 1;
        }
#pragma unroll
        for (int k = 0; k < kStages; ++k)
            if (some[k]) {
                const uint8_t *block = p.from.v + unit[k] * (32 * D);
#pragma unroll
                for (int i = 0; i < N; ++i) staged[k][i] = *reinterpret_cast<const kv_u32x4 *>(block + piece(i) * 16);
            }
    }
    __device__ __forceinline__ void load(const Sources &src, int h) {
        byte_l = p.from.vs[src.of_head(p, h)];
        int mine;
        unsigned long long starts;
        src.runs(lane, mine, starts);
        load_runs(src, h, 0, starts);
    }
    __device__ __forceinline__ void angles(const Sources &) {}
    __device__ __forceinline__ void gather(const Sources &src, int h, int next, Shelf<D> &shelf, int runs) {
        int mine;
        unsigned long long starts;
        src.runs(lane, mine, starts);
        if (half == 0 && lane < 32) {      // what the token is found by: run, slot and byte of the slot; its scale
            const int t = src.token & 31;
            shelf.spot[lane] = (uint32_t)(mine << 8 | ((2 * (t / 16) + t % 8 / 4) * 16 + 4 * (t % 16 / 8) + t % 4));
            shelf.scale[lane] = byte_scale(byte_l);
        }
        const bool whole = __builtin_amdgcn_ballot_w64(src.unit == ~0u) == 0ull && at.w.lo == 0 && at.w.hi == kKvBlock;      // every token moves
        for (int done = 0; done < runs; done += kStages) {
            if (done > 0) {
                load_runs(src, h, done, starts);
                kv_lds_barrier();      // (what lay there is picked)
            }
#pragma unroll
            for (int k = 0; k < kStages; ++k) {
                if (done + k >= runs) continue;
#pragma unroll
                for (int i = 0; i < N; ++i) *reinterpret_cast<kv_u32x4 *>(shelf.blocks + k * kStageBytes<D> + piece(i) / 4 * kStageRow + piece(i) % 4 * 16) = staged[k][i];
            }
            if (next >= 0 && done + kStages >= runs) load(src, next);      // (in flight while this head's are picked)
            kv_lds_barrier();
#pragma unroll
            for (int j0 = 0; j0 < 8; j0 += 4) {
                const uint4 spots = *reinterpret_cast<const uint4 *>(shelf.spot + token(j0));
                const float4 scales = *reinterpret_cast<const float4 *>(shelf.scale + token(j0));
                const uint32_t spot[4] = {spots.x, spots.y, spots.z, spots.w};
                const float scale[4] = {scales.x, scales.y, scales.z, scales.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int run = (int)(spot[j] >> 8) - done;
                    if (runs > kStages && (run < 0 || run >= kStages)) continue;
                    const unsigned char *tok = shelf.blocks + run * kStageBytes<D> + (spot[j] & 255u) + lane / 4 * kStageRow + half * (16 * kStageRow);
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        x[i][0][j0 + j] = code_number(tok[i * (32 * kStageRow)], scale[j]);
                        x[i][1][j0 + j] = code_number(tok[i * (32 * kStageRow) + 8], scale[j]);
                    }
                }
            }
        }
        if (whole) return;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int unit = __shfl((int)src.unit, token(j));      // (from all lanes: before any of them is left out)
            const bool moves = live(at.w, token(j)) && unit != -1;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                x[i][0][j] = moves ? x[i][0][j] : 0.f;
                x[i][1][j] = moves ? x[i][1][j] : 0.f;
            }
        }
    }
    __device__ __forceinline__ uint32_t look(const Sources &, int) {
        float all = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            top[j] = 0.f;
#pragma unroll
            for (int i = 0; i < N; ++i) top[j] = __builtin_elementwise_maximum(__builtin_elementwise_maximum(top[j], __builtin_fabsf(x[i][0][j])), __builtin_fabsf(x[i][1][j]));
            all = __builtin_elementwise_maximum(all, top[j]);
        }
        if (__builtin_amdgcn_ballot_w64(abs_bits(all) >= kInfBits) == 0ull) return 0u;
        uint32_t bad = 0u;
#pragma unroll
        for (int j = 0; j < 8; ++j) bad |= abs_bits(top[j]) >= kInfBits ? 1u << token(j) : 0u;
        return any_bits_64(bad);
    }
    __device__ __forceinline__ uint32_t largest(uint32_t bad) const {
        uint32_t m = 0u;
#pragma unroll
        for (int j = 0; j < 8; ++j) m = umax(m, (bad >> token(j)) & 1u ? 0u : abs_bits(top[j]));
        return max_bits_64(m);
    }
    __device__ __forceinline__ void write(const Target &to, const BlockScale &sc, uint32_t bad) {
        uint32_t mask[2] = {0u, 0u}, keep[2] = {0u, 0u};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (live(at.w, token(j)) && !((bad >> token(j)) & 1u)) mask[j >> 2] |= 0xffu << (8 * (j & 3));
            if (token(j) < at.w.lo) keep[j >> 2] |= 0xffu << (8 * (j & 3));
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            uint4 *dst = reinterpret_cast<uint4 *>(to.codes + piece(i) * 16);
            uint32_t v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float (&y)[8] = x[i][k >> 1];
                const int j = 4 * (k & 1);
                v[k] = codes4(y[j], y[j + 1], y[j + 2], y[j + 3], sc.scale) & mask[k & 1];
            }
            if (at.w.lo > 0) {
                const uint4 w = *reinterpret_cast<const uint4 *>(to.old + piece(i) * 16);
                const uint32_t old[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] |= (sc.grown ? kv_rescale4(old[k], sc.old_factor) : old[k]) & keep[k & 1];
            }
            *dst = make_uint4(v[0], v[1], v[2], v[3]);
        }
    }
};

template <int D, typename Side>
__device__ __forceinline__ void compact_heads(const KvCompactParams &p, const Place &at, int number, int h0, int h1, int wave, Shelf<D> &shelf, Exchange (&exchange)[2]) {
    const bool keys = wave < 2;
    const int lane = threadIdx.x & 63;
    Side side(p, at, lane, wave & 1);
    Sources src;
    src.find(p, at, h0, lane);
    const long long unit0 = kv_unit(p.to, p.batch.table, p.batch.table_width, at.sequence, h0, at.w.blk);
    if (unit0 < 0) return;      // (all wavefronts)
    side.load(src, h0);
    side.angles(src);
    for (int h = h0; h < h1; ++h) {
        const long long unit = unit0 + ((long long)(h - h0) << (p.to.page_shift - 5));
        uint8_t *codes = (keys ? p.to.k : p.to.v) + (size_t)unit * (32 * D), *byte = (keys ? p.to.ks : p.to.vs) + unit;
        Target to = {codes, byte, codes};
        if (p.stage) {
            const size_t slot = (size_t)number * p.to.heads + h;
            to.codes = p.stage + (2 * slot + (keys ? 0 : 1)) * (32 * D);
            to.byte = p.stage_bytes + 2 * slot + (keys ? 0 : 1);
        }
        const bool tells = lane == 0 && (wave & 1) == 0;      // of the side's byte, old and new
        const int held = tells && at.w.lo > 0 ? (int)*byte : 0;
        int mine;
        unsigned long long starts;
        const int next = h + 1 < h1 ? h + 1 : -1;
        side.gather(src, h, next, shelf, src.runs(lane, mine, starts));
        Exchange &ex = exchange[h & 1];      // (written again two heads on: behind a barrier that every wavefront enters when it has read it)
        const uint32_t bad = side.look(src, next), most = side.largest(bad);
        if (lane == 0) {
            ex.bad[wave] = bad;
            ex.top[wave] = most;
        }
        if (tells) ex.old_byte[wave >> 1] = held;
        kv_lds_barrier();
        const uint32_t all = ex.bad[0] | ex.bad[1] | ex.bad[2] | ex.bad[3];
        if (all != 0u) {           // (what the other side found is left out of this side's maximum too)
            kv_lds_barrier();      // the words above are read
            const uint32_t again = side.largest(all);
            if (lane == 0) ex.top[wave] = again;
            kv_lds_barrier();
        }
        const BlockScale sc = block_scale(umax(ex.top[wave & 2], ex.top[(wave & 2) + 1]), __builtin_amdgcn_readfirstlane(ex.old_byte[wave >> 1]));
        side.write(to, sc, all);
        if (tells) *to.byte = (uint8_t)sc.byte;
    }
}

template <int D>
__global__ __launch_bounds__(256, D > 128 ? 2 : D > 64 ? 4 : 5) void kv_compact_kernel(KvCompactParams p, int heads_per_wg) {
    __shared__ Exchange exchange[2];
    __shared__ Shelf<D> shelf;
    const int number = blockIdx.x;
    const Place at = place_of(p, number);
    if (at.w.lo >= at.w.hi) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h0 = blockIdx.y * heads_per_wg, h1 = h0 + heads_per_wg < p.to.heads ? h0 + heads_per_wg : p.to.heads;
    if (wave < 2) compact_heads<D, KeyMoves<D>>(p, at, number, h0, h1, wave, shelf, exchange);
    else compact_heads<D, ValueMoves<D>>(p, at, number, h0, h1, wave, shelf, exchange);
}

// Puts the blocks of the workspace in place.
template <int D>
__global__ __launch_bounds__(128) void kv_place_kernel(KvCompactParams p) {
    const Place at = place_of(p, blockIdx.x);
    if (at.w.lo >= at.w.hi) return;
    const int h = blockIdx.y, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const long long unit = kv_unit(p.to, p.batch.table, p.batch.table_width, at.sequence, h, at.w.blk);
    if (unit < 0) return;
    const size_t slot = (size_t)blockIdx.x * p.to.heads + h;
    const uint4 *src = reinterpret_cast<const uint4 *>(p.stage + (2 * slot + wave) * (32 * D));
    uint4 *dst = reinterpret_cast<uint4 *>((wave == 0 ? p.to.k : p.to.v) + (size_t)unit * (32 * D));
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
        if (wave != 0 || (lane + 64 * i) * 16 / D < at.w.hi) dst[lane + 64 * i] = src[lane + 64 * i];      // (keys behind the moves are left)
    if (lane == 0) (wave == 0 ? p.to.ks : p.to.vs)[unit] = p.stage_bytes[2 * slot + wave];
}

template <int D>
hipError_t launch_compact(const KvCompactParams &p, hipStream_t stream) {
    const int items = (int)kv_compact_items(p.batch.total, p.batch.sequences);
    // Heads a workgroup, where one list serves all: as many as leave workgroups for one round of the chip (256 CUs, four each), up to eight, so that tokens, pages and angles are looked
    // up once.  0.79 million tokens of eight heads of 128, two thirds of them kept: 762 us with two, 663 with four, 621 with eight.
    const long long rounds = (long long)items * p.to.heads / 1024;
    const int most = p.per_head || rounds < 1 ? 1 : rounds > 8 ? 8 : (int)rounds, per = most < p.to.heads ? most : p.to.heads;
    kv_compact_kernel<D><<<dim3(items, (p.to.heads + per - 1) / per), 256, 0, stream>>>(p, per);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !p.stage) return e;
    kv_place_kernel<D><<<dim3(items, p.to.heads), 128, 0, stream>>>(p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_compact(const KvCompactParams &p, hipStream_t stream) {
    switch (p.to.dim) {
        case 64: return launch_compact<64>(p, stream);
        case 128: return launch_compact<128>(p, stream);
        case 256: return launch_compact<256>(p, stream);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace svdq
