// Attention of few query rows over the paged 8-bit cache: the steps of a serving loop (layout: kv_common.h).
//
//   O_i = sum_j softmax_j(scale q'_i . k_j) v_j,   q' the rotated query, j over the keys that row i sees.
//
// The rows of a sequence and key head are its new tokens times the query heads that share the head; sixteen of them are one operand.  Keys are cut into
// chunks, a workgroup of four wavefronts has one chunk of one head, a wavefront takes every fourth block of 32 tokens: S^T = K Q^T by
// v_mfma_f32_16x16x32_f16 with the codes of the keys as exact f16 numbers (rows of the operand: tokens, in an order that makes the accumulators of
// two such products the operand of the next), the block's scale in one factor per row; running maximum and sum per row in fp32; P^T in f16;
// O^T += V^T P^T with the values as code * 2^(byte - reference), exact, the reference exponent the largest seen.  P is scaled by 2^8 (and may reach 2^14
// before the maximum is renewed), so that f16 keeps eleven bits of weights down to 2^-22 of the largest; f16 for Q, scaled by a power of two per
// row, for the same eleven bits.
// The wavefronts' sums meet in LDS.  With several chunks the parts lie in the workspace and the workgroup that finds all of its row tile arrived adds
// them in chunk order (the same bits whoever it is).
// Bound: memory, one byte per channel of a key and a value.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.h"
#include "kv_common.h"
#include "layout.h"

namespace svdq {
namespace {

constexpr float kNone = -1e30f;                  // the running maximum before the first key
constexpr float kShift = 8.f, kSlack = 6.f;      // P is exp2(t - m + kShift); m is renewed when a score passes it by kSlack
constexpr int kWaves = 4;

template <int D>
struct Block { uint4 k[2][D / 64]; uint4 v[D / 32]; uint32_t kb, vb; };      // 32 tokens of a head, as a lane holds them

template <int D>
__global__ __launch_bounds__(kWaves * 64) void kv_rows_kernel(KvAttentionParams p) {
    constexpr int C = D / 32;                    // runs of 32 channels = steps of K Q^T per 16 tokens
    constexpr int kRow = D + 4;                  // floats of a row in LDS
    __shared__ __attribute__((aligned(16))) float sums[kWaves][16][kRow];
    __shared__ float ml[kWaves][16][2];
    __shared__ float refs[kWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, q4 = lane >> 4;
    const int head = blockIdx.y, b = blockIdx.z / p.row_tiles, tile = blockIdx.z % p.row_tiles;
    int t0, n;
    kv_range(p.batch.cu, b, p.batch.total, t0, n);
    const int len = kv_length(p.cache, p.batch, b), rows = n * p.group;
    if (tile * 16 >= rows) return;
    // the lane's row and the keys [seen_lo, seen_hi) that it sees
    const int r = tile * 16 + l16 < rows ? tile * 16 + l16 : rows - 1;
    const int tok = r / p.group, qh = head * p.group + r % p.group, pos = len - n + tok;
    const int seen_hi = p.causal ? (pos + 1 < 0 ? 0 : pos + 1) : len;
    const int seen_lo = p.causal && p.window > 0 && pos + 1 > p.window ? pos + 1 - p.window : 0;
    // of the tile: its first row sees the fewest and the earliest keys
    const int tok_a = tile * 16 / p.group, last = tile * 16 + 15 < rows ? tile * 16 + 15 : rows - 1, tok_z = last / p.group;
    const int pos_a = len - n + tok_a, pos_z = len - n + tok_z;
    const int any_hi = p.causal ? (pos_z + 1 < 0 ? 0 : pos_z + 1) : len, all_hi = p.causal ? (pos_a + 1 < 0 ? 0 : pos_a + 1) : len;
    const int any_lo = p.causal && p.window > 0 && pos_a + 1 > p.window ? pos_a + 1 - p.window : 0, all_lo = p.causal && p.window > 0 && pos_z + 1 > p.window ? pos_z + 1 - p.window : 0;
    const int blk0 = any_lo >> 5, blk1 = (any_hi + 31) >> 5;
    // this workgroup's blocks
    const int chunk = blockIdx.x, count = blk1 > blk0 ? blk1 - blk0 : 0;
    int nchunks = (count + p.chunk_blocks - 1) / p.chunk_blocks;
    nchunks = nchunks < 1 ? 1 : nchunks > p.chunks ? p.chunks : nchunks;
    if (chunk >= nchunks) return;
    const int c0 = blk0 + chunk * p.chunk_blocks, c1 = chunk == nchunks - 1 ? blk1 : c0 + p.chunk_blocks;

    const int32_t *table = p.batch.table + (size_t)b * p.batch.table_width;
    const int bs = p.cache.page_shift - 5;
    auto unit_of = [&](int blk) {      // blk in [c0, c1)
        const int page = table[blk >> bs];
        return (uint32_t)page < (uint32_t)p.cache.pages ? (((long long)page * p.cache.heads + head) << bs) + (blk & ((1 << bs) - 1)) : -1ll;
    };
    auto load = [&](long long unit) {
        Block<D> t;
        const size_t u = unit < 0 ? 0 : (size_t)unit;      // (a block that the table does not name is masked)
        const uint8_t *k = p.cache.k + u * (32 * D), *v = p.cache.v + u * (32 * D);
        t.kb = p.cache.ks[u];
        t.vb = p.cache.vs[u];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int row = 16 * (l16 >> 3) + 8 * i + (l16 & 7);
#pragma unroll
            for (int c = 0; c < D / 64; ++c) t.k[i][c] = *reinterpret_cast<const uint4 *>(k + row * D + 64 * c + 16 * q4);
        }
#pragma unroll
        for (int a = 0; a < D / 32; ++a) t.v[a] = *reinterpret_cast<const uint4 *>(v + ((a * 16 + l16) * 4 + q4) * 16);
        return t;
    };
    int blk = c0 + wave;
    long long unit = -1;
    Block<D> cur;
    if (blk < c1) {
        unit = unit_of(blk);
        cur = load(unit);
    }

    // the queries: f16 of the rotated row times a power of two that brings its largest element to [2^14, 2^15)
    kv_f16x8 qf[C];
    float to_t;      // score -> exponent of 2, but for the block's scale
    {
        const uint16_t *row = p.q.data + (size_t)(t0 + tok) * p.q.token_stride + qh * p.q.head_stride;
        float x[C][8];
        uint32_t top = 0u;
#pragma unroll
        for (int c = 0; c < C; ++c) {      // step c: channels 64 (c / 2) + 16 q4 + 8 (c % 2) .. + 7
            kv_rotated8(row, p.rope, pos, 64 * (c / 2) + 16 * q4 + 8 * (c % 2), x[c]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t u = __float_as_uint(x[c][e]) & 0x7fffffffu;
                top = top > u ? top : u;
            }
        }
        const float m = kv_max32(kv_max16(__uint_as_float(top >= 0x7f800000u ? 0x7f800000u : top)));
        const int e = (int)(__float_as_uint(m) >> 23) - 127;                          // m in [2^e, 2^(e + 1))
        const int up = e < -100 ? 114 : e > 127 ? 0 : 14 - e;                         // (not finite: as it is, the row becomes NaN)
        const float f = kv_pow2(up);
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) qf[c][i] = (_Float16)(x[c][i] * f);
        to_t = p.scale * kv_pow2(-up);
    }

    kv_floatx4 o[D / 16] = {};
    float m = kNone, l = 0.f;
    int ref = 0;                                 // byte of the reference scale of the values in o

    for (; blk < c1; blk += kWaves) {
        Block<D> nxt;
        const int after = blk + kWaves;
        long long unit_next = -1;
        if (after < c1) {
            unit_next = unit_of(after);
            nxt = load(unit_next);
        }
        const int kb = __builtin_amdgcn_readfirstlane((int)cur.kb), vb = __builtin_amdgcn_readfirstlane((int)cur.vb);
        kv_floatx4 s[2] = {};
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int c = 0; c < D / 64; ++c) {
                s[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kv_f16_of(cur.k[i][c].x, cur.k[i][c].y, 1.f), qf[2 * c], s[i], 0, 0, 0);
                s[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kv_f16_of(cur.k[i][c].z, cur.k[i][c].w, 1.f), qf[2 * c + 1], s[i], 0, 0, 0);
            }
        // the lane's eight tokens are those of slot q4
        const float f = to_t * kv_pow2(kb - 127);
        float t[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] = s[j / 4][j % 4] * f;
        const bool edge = unit < 0 || blk * kKvBlock < all_lo || blk * kKvBlock + kKvBlock > all_hi;
        uint32_t live[2] = {~0u, ~0u};           // bytes of the codes of tokens that exist
        if (edge) {
            const int first = blk * kKvBlock + kv_slot_token(q4);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int key = first + (j & 3) + 8 * (j >> 2);
                const bool ok = unit >= 0 && key >= seen_lo && key < seen_hi && key < len;
                t[j] = ok ? t[j] : -__builtin_inff();
                if (unit < 0 || key >= len) live[j >> 2] &= ~(0xffu << (8 * (j & 3)));
            }
        }
        float top = t[0];
#pragma unroll
        for (int j = 1; j < 8; ++j) top = fmaxf(top, t[j]);
        top = kv_max32(kv_max16(top));
        const int ref_new = vb > ref ? vb : ref;
        if (__builtin_amdgcn_ballot_w64(top > m + kSlack) != 0ull || ref_new != ref) {
            const float m_new = fmaxf(m, top), keep = __builtin_amdgcn_exp2f(m - m_new);
            l *= keep;
            const float both = keep * kv_pow2(ref - ref_new < -126 ? -127 : ref - ref_new);
#pragma unroll
            for (int d = 0; d < D / 16; ++d) o[d] *= both;
            m = m_new;
            ref = ref_new;
        }
        kv_f16x8 pf;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float e = __builtin_amdgcn_exp2f(t[j] - m + kShift);
            l += e;
            pf[j] = (_Float16)e;
        }
        const float vf = kv_pow2(vb - ref);
#pragma unroll
        for (int a = 0; a < D / 32; ++a) {
            if (edge) {
                cur.v[a].x &= live[0]; cur.v[a].y &= live[1]; cur.v[a].z &= live[0]; cur.v[a].w &= live[1];
            }
            o[2 * a] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kv_f16_of(cur.v[a].x, cur.v[a].y, vf), pf, o[2 * a], 0, 0, 0);
            o[2 * a + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kv_f16_of(cur.v[a].z, cur.v[a].w, vf), pf, o[2 * a + 1], 0, 0, 0);
        }
        cur = nxt;
        unit = unit_next;
    }

    // ---- the wavefronts' sums meet ----
    l = kv_sum32(kv_sum16(l));
    if (q4 == 0) {
        ml[wave][l16][0] = m;
        ml[wave][l16][1] = l;
    }
    if (lane == 0) refs[wave] = (float)ref;
    __syncthreads();
    {
        float top = kNone, most = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            top = fmaxf(top, ml[w][l16][0]);
            most = fmaxf(most, refs[w]);
        }
        const float f = __builtin_amdgcn_exp2f(m - top) * kv_pow2(ref - (int)most);
#pragma unroll
        for (int d = 0; d < D / 16; ++d) *reinterpret_cast<kv_floatx4 *>(&sums[wave][l16][16 * d + 4 * q4]) = o[d] * f;
    }
    __syncthreads();
    // element (row, d) by thread; the whole block of 16 x D in 16-byte pieces
    const long long part = ((long long)blockIdx.z * p.cache.heads + head) * p.chunks;      // of this row tile's parts
    const int live_rows = rows - tile * 16 < 16 ? rows - tile * 16 : 16;
    for (int i = threadIdx.x; i < live_rows * (D / 4); i += kWaves * 64) {
        const int row = i / (D / 4), d = i % (D / 4) * 4;
        float top = kNone, most = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            top = fmaxf(top, ml[w][row][0]);
            most = fmaxf(most, refs[w]);
        }
        kv_floatx4 x = {};
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            x += *reinterpret_cast<const kv_floatx4 *>(&sums[w][row][d]);
            sum += ml[w][row][1] * __builtin_amdgcn_exp2f(ml[w][row][0] - top);
        }
        x *= kv_pow2((int)most - 127);
        if (nchunks > 1) {      // past the L2 of this XCD: the workgroup that adds the parts may run on another
            float *dst = p.partial + ((part + chunk) * 16 + row) * D + d;
#pragma unroll
            for (int k = 0; k < 4; ++k) __hip_atomic_store(dst + k, x[k], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            if (d == 0) {
                float *q = p.partial_ml + ((part + chunk) * 16 + row) * 2;
                __hip_atomic_store(q, top, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                __hip_atomic_store(q + 1, sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
        } else {
            const float inv = sum > 0.f ? 1.f / sum : sum == sum ? 0.f : sum;      // (no key seen: zeros)
            const int rr = tile * 16 + row;
            uint16_t *dst = p.out + ((size_t)(t0 + rr / p.group) * p.q_heads + head * p.group + rr % p.group) * D + d;
            const kv_bf16x2 lo = {(__bf16)(x[0] * inv), (__bf16)(x[1] * inv)}, hi = {(__bf16)(x[2] * inv), (__bf16)(x[3] * inv)};
            *reinterpret_cast<uint2 *>(dst) = make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
        }
    }
    if (nchunks == 1) return;

    // ---- the parts of the row tile meet: the arrival words hold anything but kKvArrived until a workgroup marks its own, and are cleared at the end ----
    __shared__ int everyone;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) everyone = 1;
    __syncthreads();
    unsigned long long *words = p.arrived + part;
    if (threadIdx.x == 0) {
        (void)__hip_atomic_exchange(words + chunk, kKvArrived, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < nchunks; i += kWaves * 64)
        if (__hip_atomic_load(words + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != kKvArrived) everyone = 0;
    __syncthreads();
    if (!everyone) return;
    for (int i = threadIdx.x; i < live_rows * (D / 4); i += kWaves * 64) {
        const int row = i / (D / 4), d = i % (D / 4) * 4;
        float top = kNone, sum = 0.f;
        kv_floatx4 x = {};
        for (int c = 0; c < nchunks; ++c) {
            const float *q = p.partial_ml + ((part + c) * 16 + row) * 2, *src = p.partial + ((part + c) * 16 + row) * D + d;
            const float mc = __hip_atomic_load(q, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT), lc = __hip_atomic_load(q + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            kv_floatx4 y;
#pragma unroll
            for (int k = 0; k < 4; ++k) y[k] = __hip_atomic_load(src + k, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            const float m_new = fmaxf(top, mc), f = __builtin_amdgcn_exp2f(top - m_new), g = __builtin_amdgcn_exp2f(mc - m_new);
            x = x * f + y * g;
            sum = sum * f + lc * g;
            top = m_new;
        }
        const float inv = sum > 0.f ? 1.f / sum : sum == sum ? 0.f : sum;
        const int rr = tile * 16 + row;
        uint16_t *dst = p.out + ((size_t)(t0 + rr / p.group) * p.q_heads + head * p.group + rr % p.group) * D + d;
        const kv_bf16x2 lo = {(__bf16)(x[0] * inv), (__bf16)(x[1] * inv)}, hi = {(__bf16)(x[2] * inv), (__bf16)(x[3] * inv)};
        *reinterpret_cast<uint2 *>(dst) = make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
    }
    // (every workgroup of the row tile has made its mark; two that both found all marks store the same results)
    for (int i = threadIdx.x; i < nchunks; i += kWaves * 64) __hip_atomic_store(words + i, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

}  // namespace

hipError_t launch_kv_attention_rows(const KvAttentionParams &p, hipStream_t stream) {
    const dim3 grid(p.chunks, p.cache.heads, p.batch.sequences * p.row_tiles);
    switch (p.cache.dim) {
        case 64: kv_rows_kernel<64><<<grid, kWaves * 64, 0, stream>>>(p); break;
        case 128: kv_rows_kernel<128><<<grid, kWaves * 64, 0, stream>>>(p); break;
        case 256: kv_rows_kernel<256><<<grid, kWaves * 64, 0, stream>>>(p); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

}  // namespace svdq
