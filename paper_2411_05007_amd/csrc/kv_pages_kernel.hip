// Pages of the paged 8-bit cache (layout: kv_common.h) that several sequences share: counts and block tables on the GPU, so that a step needs no look at lengths by the host.
//
// refs[p] counts the table entries that name page p; none: the page is free.
//   fork      a row of a table becomes the pages of another row's tokens; their counts go up
//   release   entries of pages wholly within a range of tokens are cleared; their counts go down
//   reserve   every entry that a batch's new tokens fall in names a page of the sequence's own: entries that name none, or one with a count above one, get the lowest free pages, in the
//             order of sequences and entries, and what a shared page held before the new tokens is copied.  Where all the entries that name a page are to leave it, the first sequence
//             keeps it.  A sequence's first entry that names none while tokens before the new ones fall in it (they found no page, or it was given back) gets none: nothing could
//             fill those tokens' places, and another sequence's would be seen there
//   copy      pages of one cache into pages of the same or another one
// Reserve is two kernels.  The first notes what is free (a bit a page, counts for each 1024) and which entries lack a page (a bit an entry, a count for each sequence), the second
// sums what comes before its sequence, enumerates the free pages from there and the entries side by side through LDS, and writes table and counts; further workgroups of the
// sequence find the one page that they copy to by themselves.  Decisions are made from the first one's notes alone, so the order in which workgroups change tables and counts does not matter.
// Bound: latency, of two launches; then memory, for the copies.  32 branches of eight sequences: release 2.3, fork 2.6, notes 3.5 (3.2 without the search for a shared page's last holders), reserve
// 4.7 us with 5.9 MB read and written (16.4 where every step of the search waited for the one before); 256 branches, pages of 256: 4.0, 3.4, 4.4 (3.2; 5.7 with 64 sequences asked for at a time) and
// 16 us, in which 80 MB pass the L2s, 5.0 TB/s.  40 of those are reads, though the pages that four branches share are 10: the four are on different XCDs, and each L2 fetches its own.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.h"
#include "kv_common.h"

namespace svdq {
namespace {

__device__ __forceinline__ bool is_page(int page, int pages) { return (uint32_t)page < (uint32_t)pages; }
__device__ __forceinline__ void count_by(int32_t *refs, int by) { (void)__hip_atomic_fetch_add(refs, by, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

__global__ __launch_bounds__(256) void kv_release_kernel(KvPool pool, int32_t *table, const int32_t *first, const int32_t *last, int width) {
    const int b = blockIdx.y, e = (int)(blockIdx.x * 256 + threadIdx.x);
    if (e >= width) return;
    const size_t i = (size_t)b * width + e;
    const long long lo = first ? first[b] : 0, hi = last ? (long long)last[b] : 1ll << 62;
    if (((long long)e << pool.page_shift) < lo || ((long long)(e + 1) << pool.page_shift) > hi) return;
    const int page = table[i];
    if (is_page(page, pool.pages)) count_by(pool.refs + page, -1);
    table[i] = -1;
}

__global__ __launch_bounds__(256) void kv_fork_kernel(KvForkParams p) {
    const int b = blockIdx.y, e = (int)(blockIdx.x * 256 + threadIdx.x);
    if (e >= p.to_width) return;
    const int from = p.parent[b];
    int len = 0, page = -1;
    if ((uint32_t)from < (uint32_t)p.from_sequences) {
        const long long most = (long long)(p.from_width < p.to_width ? p.from_width : p.to_width) << p.pool.page_shift;
        len = p.from_len[from];
        len = len < 0 ? 0 : (long long)len > most ? (int)most : len;
        if (((long long)e << p.pool.page_shift) < len) page = p.from_table[(size_t)from * p.from_width + e];
    }
    if (!is_page(page, p.pool.pages)) page = -1;
    else count_by(p.pool.refs + page, 1);
    p.to_table[(size_t)b * p.to_width + e] = page;
    if (e == 0) p.to_len[b] = len;
}

// ---- reserve ----------------------------------------------------------------------------------------------------------------
constexpr int kSlicePages = 1024;      // pages of a count
constexpr int kLost = -2;              // in the place of a shared page: the first entry is to stay without one
struct Entries { int lo, hi, before; };      // of a sequence's table that its new tokens fall in; tokens before them
__device__ __forceinline__ Entries entries_between(const KvReserveParams &p, int cu0, int cu1, int len) {
    const int t0 = kv_within(cu0, 0, p.batch.total), n = kv_within(cu1, t0, p.batch.total) - t0;
    const long long most = (long long)p.batch.table_width << p.pool.page_shift;
    len = len < 0 ? 0 : (long long)len > most ? (int)most : len;
    const int before = len > n ? len - n : 0;
    Entries e = {before >> p.pool.page_shift, (int)(((long long)len + (1 << p.pool.page_shift) - 1) >> p.pool.page_shift), before};
    if (n == 0 || e.hi < e.lo) e.hi = e.lo;
    return e;
}
__device__ __forceinline__ Entries entries_of(const KvReserveParams &p, int b) {      // b the same in all lanes
    return entries_between(p, __builtin_amdgcn_readfirstlane(p.batch.cu[b]), __builtin_amdgcn_readfirstlane(p.batch.cu[b + 1]), __builtin_amdgcn_readfirstlane(p.batch.kv_len[b]));
}
__device__ __forceinline__ int wave_sum(int x) { return __builtin_amdgcn_readlane(kv_sum_upto(x), 63); }

__global__ __launch_bounds__(256) void kv_reserve_plan_kernel(KvReserveParams p) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if ((int)blockIdx.x < p.slices) {      // free pages
        __shared__ int counts[4];
        int count = 0;
        int refs[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int page = (int)blockIdx.x * kSlicePages + (4 * wave + i) * 64 + lane;
            refs[i] = page < p.pool.pages ? p.pool.refs[page] : 1;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned long long word = __builtin_amdgcn_ballot_w64(refs[i] <= 0);
            if (lane == 0) p.free_words[(int)blockIdx.x * (kSlicePages / 64) + 4 * wave + i] = word;
            count += __builtin_popcountll(word);
        }
        if (lane == 0) counts[wave] = count;
        __syncthreads();
        if (threadIdx.x == 0) p.slice_free[blockIdx.x] = counts[0] + counts[1] + counts[2] + counts[3];
        return;
    }
    const int b = ((int)blockIdx.x - p.slices) * 4 + wave;      // entries that lack a page
    if (b >= p.batch.sequences) return;
    // A page that a sequence would leave is looked for in the same entry of the others (a branch has it where its parent does), 64 of them at a time: the first 64 are asked for in time.
    const int last = p.batch.sequences - 1;
    struct Peer { int cu0, cu1, len, page; };
    const auto ask = [&](int j, int e) { return Peer{p.batch.cu[j], p.batch.cu[j + 1], p.batch.kv_len[j], p.batch.table[(size_t)j * p.batch.table_width + e]}; };
    const Entries at = entries_of(p, b);
    const Peer first_peer = ask(lane < last ? lane : last, at.lo < at.hi ? at.lo : 0);
    // The batch has all the entries that name the page, and b is the first sequence of them: it keeps the page.
    const auto keeps = [&](int e, int page, int count) {
        if (count > p.batch.sequences) return false;
        int found = 0, first = -1;
        const auto look = [&](const Peer &x, int j0) {
            const Entries others = entries_between(p, x.cu0, x.cu1, x.len);
            const unsigned long long word = __builtin_amdgcn_ballot_w64(j0 + lane <= last && e >= others.lo && e < others.hi && x.page == page);
            if (first < 0 && word != 0ull) first = j0 + __builtin_ctzll(word);
            found += __builtin_popcountll(word);
        };
        int j0 = 0;
        if (e == at.lo) {
            look(first_peer, 0);
            j0 = 64;
        }
        constexpr int kAhead = 4;
        for (; j0 <= last && (first < 0 || first == b); j0 += 64 * kAhead) {
            Peer x[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) x[i] = ask(j0 + 64 * i + lane < last ? j0 + 64 * i + lane : last, e);
#pragma unroll
            for (int i = 0; i < kAhead; ++i) look(x[i], j0 + 64 * i);
        }
        return first == b && found == count;
    };
    const bool holds = (long long)at.lo << p.pool.page_shift < at.before;      // tokens before the new ones fall in the first entry
    int count = 0, shared = -1;
    for (int e0 = at.lo & ~63; e0 < at.hi; e0 += 64) {
        const int e = e0 + lane;
        bool lacks = e >= at.lo && e < at.hi;
        const int page = lacks ? p.batch.table[(size_t)b * p.batch.table_width + e] : -1;
        const bool named = is_page(page, p.pool.pages);
        const int refs = named ? p.pool.refs[page] : 0;
        if (named) lacks = refs > 1;
        for (unsigned long long left = __builtin_amdgcn_ballot_w64(named && lacks); left != 0ull; left &= left - 1) {
            const int i = __builtin_ctzll(left);
            if (keeps(e0 + i, __builtin_amdgcn_readlane(page, i), __builtin_amdgcn_readlane(refs, i)) && lane == i) lacks = false;
        }
        const bool lost = lacks && !named && holds && e == at.lo;
        lacks = lacks && !lost;
        if (__builtin_amdgcn_ballot_w64(lost) != 0ull) shared = kLost;
        const unsigned long long word = __builtin_amdgcn_ballot_w64(lacks);
        if (lane == 0) p.lacks[(size_t)b * p.words + (e0 >> 6)] = word;
        count += __builtin_popcountll(word);
        if (e0 <= at.lo && at.lo < e0 + 64) {      // (what the first entry holds before the new tokens)
            const int first = __builtin_amdgcn_readlane(lacks && named ? page : -1, at.lo - e0);
            if (holds && shared != kLost) shared = first;
        }
    }
    if (lane == 0) {
        p.lack_count[b] = count;
        p.shared[b] = shared;
    }
}

// Copies the blocks of a page's first tokens, part `part` of `parts` of it (a workgroup of 256): the keys and values of a head lie in a row, and go in chunks of 16 KB.
__device__ __forceinline__ void copy_page(const KvCache &to, const KvCache &from, int to_page, int from_page, int tokens, int part, int parts) {
    const int bs = to.page_shift - 5, most = 32 << bs, blocks = ((tokens < most ? tokens : most) + 31) >> 5;
    if (blocks <= 0) return;
    constexpr int kAhead = 4, kChunk = 256 * kAhead;
    const int pieces = blocks * 2 * to.dim, chunks = (pieces + kChunk - 1) / kChunk, items = to.heads * 2 * chunks;      // pieces of 16 bytes of a head's keys, or values
    const size_t to_unit = ((size_t)to_page * to.heads) << bs, from_unit = ((size_t)from_page * to.heads) << bs;
    for (int item = part; item < items; item += parts) {
        const int side = item / chunks, at = item % chunks * kChunk + (int)threadIdx.x;
        const size_t head = (size_t)(side >> 1) << bs;
        const kv_u32x4 *src = reinterpret_cast<const kv_u32x4 *>((side & 1 ? from.v : from.k) + (from_unit + head) * (32 * (size_t)to.dim));
        kv_u32x4 *dst = reinterpret_cast<kv_u32x4 *>((side & 1 ? to.v : to.k) + (to_unit + head) * (32 * (size_t)to.dim));
        kv_u32x4 w[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) w[k] = src[at + 256 * k < pieces ? at + 256 * k : pieces - 1];
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (at + 256 * k < pieces) dst[at + 256 * k] = w[k];
    }
    if (part == 0)
        for (int i = threadIdx.x; i < to.heads * blocks; i += 256) {
            const size_t at = ((size_t)(i / blocks) << bs) + i % blocks;
            to.ks[to_unit + at] = from.ks[from_unit + at];
            to.vs[to_unit + at] = from.vs[from_unit + at];
        }
}

// What a wavefront of a sequence needs of the first kernel's notes, asked for at once: the entries that lack a page in sequences before `b`, the free pages of the first 64 slices (one in
// a lane) and the first 64 words of their bits.
struct Notes {
    int before, slice_l;
    unsigned long long word_l;
    __device__ __forceinline__ void read(const KvReserveParams &p, int b) {
        const int lane = threadIdx.x & 63;
        slice_l = lane < p.slices ? p.slice_free[lane] : 0;
        word_l = p.free_words[lane < p.slices * (kSlicePages / 64) ? lane : 0];
        int sum = 0;
#pragma unroll 4
        for (int i = lane; i < b; i += 64) sum += p.lack_count[i];
        before = wave_sum(sum);
    }
};
// Free pages in order, from the `skip`-th on, up to `most` of them into `out`; returns how many there were.
__device__ __forceinline__ int free_pages(const KvReserveParams &p, const Notes &notes, int skip, int most, int *out) {
    const int lane = threadIdx.x & 63, words = p.slices * (kSlicePages / 64);
    int s0 = 0;
    if (p.slices > 4)
        for (; s0 < p.slices; s0 += 64) {      // the slice that has it
            const int mine = s0 == 0 ? notes.slice_l : s0 + lane < p.slices ? p.slice_free[s0 + lane] : 0, upto = kv_sum_upto(mine);
            const unsigned long long past = __builtin_amdgcn_ballot_w64(upto > skip);
            if (past != 0ull) {
                const int at = __builtin_ctzll(past);
                skip -= __builtin_amdgcn_readlane(upto - mine, at);
                s0 += at;
                break;
            }
            skip -= __builtin_amdgcn_readlane(upto, 63);
        }
    int got = 0;
    for (int w0 = s0 * (kSlicePages / 64); w0 < words && got < most; w0 += 64) {      // 64 words at a time, one in a lane
        unsigned long long word = w0 == 0 ? notes.word_l : w0 + lane < words ? p.free_words[w0 + lane] : 0ull;
        if (w0 + lane >= words) word = 0ull;
        const int here = __builtin_popcountll(word), upto = kv_sum_upto(here);
        unsigned long long left = __builtin_amdgcn_ballot_w64(here > 0 && upto > skip);      // words that still matter, one after the other: a page in a lane
        for (; left != 0ull && got < most; left &= left - 1) {
            const int at = __builtin_ctzll(left);
            const unsigned long long bits = ((unsigned long long)(uint32_t)__builtin_amdgcn_readlane((int)(word >> 32), at) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)word, at);
            const int first = __builtin_amdgcn_readlane(upto - here, at), number = first + __builtin_popcountll(bits & ((1ull << lane) - 1ull)) - skip + got;
            if (((bits >> lane) & 1ull) && number >= got && number < most) out[number] = (w0 + at) * 64 + lane;
            const int end = first + __builtin_popcountll(bits), taken = end - skip;      // (at least one)
            got = got + taken < most ? got + taken : most;
            skip = end;
        }
        const int total = __builtin_amdgcn_readlane(upto, 63);
        skip = skip > total ? skip - total : 0;
    }
    return got;
}

// Part 0 of a sequence writes tables and counts, the others copy.
__global__ __launch_bounds__(256) void kv_reserve_kernel(KvReserveParams p) {
    constexpr int kRound = 256;
    __shared__ int pages[kRound], entry[kRound], target_of[4], found;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), b = blockIdx.x, part = blockIdx.y;
    const int count = p.lack_count[b], shared = p.shared[b];
    if (part > 0) {
        Notes notes;
        notes.read(p, b);
        const Entries at = entries_of(p, b);
        if (shared < 0) return;
        if (free_pages(p, notes, notes.before, 1, target_of + wave) == 0) return;      // (the same in all wavefronts)
        __builtin_amdgcn_wave_barrier();
        const int target = __builtin_amdgcn_readfirstlane(*(volatile int *)(target_of + wave));
        copy_page(p.cache, p.cache, target, shared, at.before - (at.lo << p.pool.page_shift), part - 1, (int)gridDim.y - 1);
        return;
    }
    if (b == 0 && wave == 3 && p.missing) {      // entries that lack a page, in all, and free pages; entries that get none
        int lack = 0, lost = 0;
        for (int i = lane; i < p.batch.sequences; i += 64) {
            lack += p.lack_count[i];
            lost += p.shared[i] == kLost ? 1 : 0;
        }
        for (int i = lane; i < p.slices; i += 64) lack -= p.slice_free[i];
        lack = wave_sum(lack);
        lost = wave_sum(lost);
        if (lane == 0) *p.missing = (lack > 0 ? lack : 0) + lost;
    }
    int target = -1;      // of the copy: the first page
    if (count > 0) {
        Notes notes;
        notes.read(p, b);
        const Entries at = entries_of(p, b);
        for (int done = 0; done < count; done += kRound) {
            const int round = count - done < kRound ? count - done : kRound;
            if (wave == 0) {
                const int n = free_pages(p, notes, notes.before + done, round, pages);
                if (lane == 0) found = n;
            } else if (wave == 1) {      // the entries of this round, from where the last one ended
                int got = 0, skip = done;
                for (int e = at.lo & ~63; e < at.hi && got < round; e += 64) {
                    const unsigned long long word = p.lacks[(size_t)b * p.words + (e >> 6)];
                    const int total = __builtin_popcountll(word), number = __builtin_popcountll(word & ((1ull << lane) - 1ull)) - skip + got;
                    if (((word >> lane) & 1ull) && number >= got && number < round) entry[number] = e + lane;
                    const int taken = total > skip ? total - skip : 0;
                    got = got + taken < round ? got + taken : round;
                    skip = skip > total ? skip - total : 0;
                }
            }
            __syncthreads();
            if (done == 0) target = found > 0 ? pages[0] : -1;
            if ((int)threadIdx.x < round) {
                int32_t *at_entry = const_cast<int32_t *>(p.batch.table) + (size_t)b * p.batch.table_width + entry[threadIdx.x];
                const int old = *at_entry, page = (int)threadIdx.x < found ? pages[threadIdx.x] : -1;
                if (is_page(old, p.pool.pages)) count_by(p.pool.refs + old, -1);
                if (page >= 0) p.pool.refs[page] = 1;
                *at_entry = page;
            }
            __syncthreads();
        }
        if (p.copies && threadIdx.x < 3) {
            const bool any = shared >= 0 && target >= 0;
            p.copies[3 * b + threadIdx.x] = threadIdx.x == 0 ? any ? shared : -1 : threadIdx.x == 1 ? any ? target : -1 : any ? at.before - (at.lo << p.pool.page_shift) : 0;
        }
        return;
    }
    if (p.copies && threadIdx.x < 3) p.copies[3 * b + threadIdx.x] = threadIdx.x < 2 ? -1 : 0;
}

__global__ __launch_bounds__(256) void kv_copy_pages_kernel(KvCache to, KvCache from, const int32_t *copies) {
    const int32_t *c = copies + 3 * (size_t)blockIdx.x;
    const int from_page = c[0], to_page = c[1], tokens = c[2];
    if (!is_page(from_page, from.pages) || !is_page(to_page, to.pages) || tokens <= 0) return;
    copy_page(to, from, to_page, from_page, tokens, blockIdx.y, gridDim.y);
}

__global__ void kv_none_missing_kernel(int32_t *missing) { *missing = 0; }

// Workgroups of a copy: one for each 16 KB of a head's keys or values, but no more than fill the chip twice (256 CUs, eight each).
int copy_parts(long long copies, const KvCache &c) {
    const long long chunks = (((long long)c.dim << c.page_shift) + 16383) / 16384, most = chunks * 2 * c.heads, room = 4096 / (copies < 1 ? 1 : copies), n = room < most ? room : most;
    return n < 1 ? 1 : n > 65000 ? 65000 : (int)n;
}

}  // namespace

KvReservePlan plan_kv_reserve(int pages, int sequences, int width) {
    KvReservePlan r{};
    const auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    r.slices = (int)(((long long)pages + kSlicePages - 1) / kSlicePages);
    r.words = (int)(((long long)width + 63) / 64);
    r.slice_off = up((size_t)r.slices * (kSlicePages / 64) * 8);
    r.count_off = r.slice_off + up((size_t)r.slices * 4);
    r.shared_off = r.count_off + up((size_t)sequences * 4);
    r.lacks_off = r.shared_off + up((size_t)sequences * 4);
    r.total = r.lacks_off + up((size_t)sequences * r.words * 8);
    return r;
}

hipError_t launch_kv_release(const KvPool &pool, int32_t *table, const int32_t *first, const int32_t *last, int sequences, int width, hipStream_t stream) {
    kv_release_kernel<<<dim3((width + 255) / 256, sequences), 256, 0, stream>>>(pool, table, first, last, width);
    return hipGetLastError();
}
hipError_t launch_kv_fork(const KvForkParams &p, hipStream_t stream) {
    kv_fork_kernel<<<dim3((p.to_width + 255) / 256, p.sequences), 256, 0, stream>>>(p);
    return hipGetLastError();
}
hipError_t launch_kv_reserve(const KvReserveParams &p, hipStream_t stream) {
    if (p.batch.sequences == 0) {
        kv_none_missing_kernel<<<1, 1, 0, stream>>>(p.missing);
        return hipGetLastError();
    }
    kv_reserve_plan_kernel<<<p.slices + (p.batch.sequences + 3) / 4, 256, 0, stream>>>(p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    kv_reserve_kernel<<<dim3(p.batch.sequences, p.cache.k ? 1 + copy_parts(p.batch.sequences, p.cache) : 1), 256, 0, stream>>>(p);
    return hipGetLastError();
}
hipError_t launch_kv_copy_pages(const KvCache &to, const KvCache &from, const int32_t *copies, int n, hipStream_t stream) {
    kv_copy_pages_kernel<<<dim3(n, copy_parts(n, to)), 256, 0, stream>>>(to, from, copies);
    return hipGetLastError();
}

}  // namespace svdq
