// Pages of the paged 8-bit cache (layout: kv_common.h) that several sequences share: counts and block tables on the GPU, so that a step needs no look at lengths by the host.
//
// refs[p] counts the table entries that name page p; none: the page is free.
//   fork      a row of a table becomes the pages of another row's tokens; their counts go up
//   release   entries of pages wholly within a range of tokens are cleared; their counts go down
//   reserve   every entry that a batch's new tokens fall in names a page of the sequence's own: entries that name none, or one with a count above one, get the lowest free pages, in the
//             order of sequences and entries, and what a shared page held before the new tokens is copied
//   copy      pages of one cache into pages of the same or another one
// Reserve is two kernels.  The first notes what is free (a bit a page, counts for each 1024) and which entries lack a page (a bit an entry, a count for each sequence), the second
// sums what comes before its sequence, enumerates the free pages from there and the entries side by side through LDS, and writes table and counts; further workgroups of the
// sequence copy.  Decisions are made from the first one's notes alone, so the order in which workgroups change tables and counts does not matter.
// Bound: latency, of two launches; then memory, for the copies.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.h"
#include "kv_common.h"

namespace svdq {
namespace {

__device__ __forceinline__ bool is_page(int page, int pages) { return (uint32_t)page < (uint32_t)pages; }
__device__ __forceinline__ void count_by(int32_t *refs, int by) { (void)__hip_atomic_fetch_add(refs, by, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

__global__ __launch_bounds__(256) void kv_release_kernel(KvPool pool, int32_t *table, const int32_t *first, const int32_t *last, int sequences, int width) {
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i >= (long long)sequences * width) return;
    const int b = (int)(i / width), e = (int)(i % width);
    const long long lo = first ? first[b] : 0, hi = last ? (long long)last[b] : 1ll << 62;
    if (((long long)e << pool.page_shift) < lo || ((long long)(e + 1) << pool.page_shift) > hi) return;
    const int page = table[i];
    if (is_page(page, pool.pages)) count_by(pool.refs + page, -1);
    table[i] = -1;
}

__global__ __launch_bounds__(256) void kv_fork_kernel(KvForkParams p) {
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i >= (long long)p.sequences * p.to_width) return;
    const int b = (int)(i / p.to_width), e = (int)(i % p.to_width), from = p.parent[b];
    int len = 0, page = -1;
    if ((uint32_t)from < (uint32_t)p.from_sequences) {
        const long long most = (long long)(p.from_width < p.to_width ? p.from_width : p.to_width) << p.pool.page_shift;
        len = p.from_len[from];
        len = len < 0 ? 0 : (long long)len > most ? (int)most : len;
        if (((long long)e << p.pool.page_shift) < len) page = p.from_table[(size_t)from * p.from_width + e];
    }
    if (!is_page(page, p.pool.pages)) page = -1;
    else count_by(p.pool.refs + page, 1);
    p.to_table[i] = page;
    if (e == 0) p.to_len[b] = len;
}

// ---- reserve ----------------------------------------------------------------------------------------------------------------
constexpr int kSlicePages = 1024;      // pages of a count
struct Entries { int lo, hi, before; };      // of a sequence's table that its new tokens fall in; tokens before them
__device__ __forceinline__ Entries entries_of(const KvReserveParams &p, int b) {
    int t0, n;
    kv_range(p.batch.cu, b, p.batch.total, t0, n);
    const long long most = (long long)p.batch.table_width << p.pool.page_shift;
    int len = __builtin_amdgcn_readfirstlane(p.batch.kv_len[b]);
    len = len < 0 ? 0 : (long long)len > most ? (int)most : len;
    const int before = len > n ? len - n : 0;
    Entries e = {before >> p.pool.page_shift, (int)(((long long)len + (1 << p.pool.page_shift) - 1) >> p.pool.page_shift), before};
    if (n == 0 || e.hi < e.lo) e.hi = e.lo;
    return e;
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
    const Entries at = entries_of(p, b);
    int count = 0, shared = -1;
    for (int e0 = at.lo & ~63; e0 < at.hi; e0 += 64) {
        const int e = e0 + lane;
        bool lacks = e >= at.lo && e < at.hi;
        const int page = lacks ? p.batch.table[(size_t)b * p.batch.table_width + e] : -1;
        const bool named = is_page(page, p.pool.pages);
        if (named) lacks = p.pool.refs[page] > 1;
        const unsigned long long word = __builtin_amdgcn_ballot_w64(lacks);
        if (lane == 0) p.lacks[(size_t)b * p.words + (e0 >> 6)] = word;
        count += __builtin_popcountll(word);
        if (e0 <= at.lo && at.lo < e0 + 64) {      // (what the first entry holds before the new tokens)
            const int first = __builtin_amdgcn_readlane(lacks && named ? page : -1, at.lo - e0);
            if ((long long)at.lo << p.pool.page_shift < at.before) shared = first;
        }
    }
    if (lane == 0) {
        p.lack_count[b] = count;
        p.shared[b] = shared;
    }
}

// Copies the blocks of a page's first tokens, part `part` of `parts` of it (a workgroup of 256).
__device__ __forceinline__ void copy_page(const KvCache &to, const KvCache &from, int to_page, int from_page, int tokens, int part, int parts) {
    const int bs = to.page_shift - 5, most = 1 << bs, blocks = (tokens + 31) >> 5 < most ? (tokens + 31) >> 5 : most;
    if (blocks <= 0) return;
    const int per = blocks * 2 * to.dim, total = to.heads * 2 * per;      // pieces of 16 bytes of a head's keys or values, of all
    const size_t to_unit = ((size_t)to_page * to.heads) << bs, from_unit = ((size_t)from_page * to.heads) << bs;
    const auto src = [&](int i) {
        const int side = i / per, h = side >> 1;
        return reinterpret_cast<const uint4 *>((side & 1 ? from.v : from.k) + (from_unit + ((size_t)h << bs)) * (32 * (size_t)to.dim)) + i % per;
    };
    const auto dst = [&](int i) {
        const int side = i / per, h = side >> 1;
        return reinterpret_cast<uint4 *>((side & 1 ? to.v : to.k) + (to_unit + ((size_t)h << bs)) * (32 * (size_t)to.dim)) + i % per;
    };
    constexpr int kAhead = 4;
    for (int i0 = part * 256 * kAhead; i0 < total; i0 += parts * 256 * kAhead) {
        uint4 w[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int i = i0 + 256 * k + threadIdx.x;
            w[k] = *src(i < total ? i : total - 1);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int i = i0 + 256 * k + threadIdx.x;
            if (i < total) *dst(i) = w[k];
        }
    }
    if (part == 0)
        for (int i = threadIdx.x; i < to.heads * blocks; i += 256) {
            const size_t at = ((size_t)(i / blocks) << bs) + i % blocks;
            to.ks[to_unit + at] = from.ks[from_unit + at];
            to.vs[to_unit + at] = from.vs[from_unit + at];
        }
}

// Free pages in order, from the `skip`-th on, up to `most` of them into `out` (a wavefront); returns how many there were.
__device__ __forceinline__ int free_pages(const KvReserveParams &p, int skip, int most, int *out) {
    const int lane = threadIdx.x & 63;
    int s0 = 0, got = 0;
    for (; s0 < p.slices; s0 += 64) {      // the slice that has it
        const int mine = s0 + lane < p.slices ? p.slice_free[s0 + lane] : 0, upto = kv_sum_upto(mine);
        const unsigned long long past = __builtin_amdgcn_ballot_w64(upto > skip);
        if (past != 0ull) {
            const int at = __builtin_ctzll(past);
            skip -= __builtin_amdgcn_readlane(upto - mine, at);
            s0 += at;
            break;
        }
        skip -= __builtin_amdgcn_readlane(upto, 63);
    }
    const int words = p.slices * (kSlicePages / 64);
    for (int w0 = s0 * (kSlicePages / 64); w0 < words && got < most; w0 += 64) {      // 64 words at a time
        const unsigned long long word = w0 + lane < words ? p.free_words[w0 + lane] : 0ull;
        const int here = __builtin_popcountll(word), upto = kv_sum_upto(here), total = __builtin_amdgcn_readlane(upto, 63);
        // the lane's pages have the numbers upto - here .. upto - 1; those from `skip` on are taken
        int number = upto - here - skip + got;
        for (unsigned long long left = word; left != 0ull && number < most; left &= left - 1, ++number)
            if (number >= got) out[number] = (w0 + lane) * 64 + __builtin_ctzll(left);
        const int taken = total > skip ? total - skip : 0;
        got = got + taken < most ? got + taken : most;
        skip = skip > total ? skip - total : 0;
    }
    return got;
}

__global__ __launch_bounds__(256) void kv_reserve_kernel(KvReserveParams p) {
    constexpr int kRound = 256;
    __shared__ int pages[kRound], entry[kRound], sums[3][4];
    __shared__ int found;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), b = blockIdx.x, part = blockIdx.y;
    const bool writes = part == 0, first_of_all = b == 0 && writes;
    const int count = p.lack_count[b], shared = p.shared[b];
    if (!first_of_all && (writes ? count == 0 && !p.copies : shared < 0 || !p.cache.k)) return;
    // entries that lack a page in sequences before this one (and, for one workgroup, in all; and the free pages)
    int before = 0, all = 0, free = 0;
    const int last = first_of_all ? p.batch.sequences : b;
    for (int i = threadIdx.x; i < last; i += 256) {
        const int n = p.lack_count[i];
        before += i < b ? n : 0;
        all += n;
    }
    if (first_of_all)
        for (int i = threadIdx.x; i < p.slices; i += 256) free += p.slice_free[i];
    before = wave_sum(before);
    all = wave_sum(all);
    free = wave_sum(free);
    if (lane == 0) {
        sums[0][wave] = before;
        sums[1][wave] = all;
        sums[2][wave] = free;
    }
    __syncthreads();
    before = sums[0][0] + sums[0][1] + sums[0][2] + sums[0][3];
    if (first_of_all && threadIdx.x == 0 && p.missing) {
        const int lack = sums[1][0] + sums[1][1] + sums[1][2] + sums[1][3] - (sums[2][0] + sums[2][1] + sums[2][2] + sums[2][3]);
        *p.missing = lack > 0 ? lack : 0;
    }
    if (count == 0) {
        if (writes && p.copies && threadIdx.x < 3) p.copies[3 * b + threadIdx.x] = threadIdx.x < 2 ? -1 : 0;
        return;
    }
    const Entries at = entries_of(p, b);
    const int held = at.before - (at.lo << p.pool.page_shift);      // tokens of a shared page before the new ones
    int target = -1;      // of the copy: the first page
    for (int done = 0; done < count; done += kRound) {
        const int round = writes ? (count - done < kRound ? count - done : kRound) : 1;
        if (wave == 0) {
            const int n = free_pages(p, before + done, round, pages);
            if (lane == 0) found = n;
        } else if (wave == 1 && writes) {      // the entries of this round, from where the last one ended
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
        if (!writes) break;
        if ((int)threadIdx.x < round) {
            int32_t *at_entry = const_cast<int32_t *>(p.batch.table) + (size_t)b * p.batch.table_width + entry[threadIdx.x];
            const int old = *at_entry, page = (int)threadIdx.x < found ? pages[threadIdx.x] : -1;
            if (is_page(old, p.pool.pages)) count_by(p.pool.refs + old, -1);
            if (page >= 0) p.pool.refs[page] = 1;
            *at_entry = page;
        }
        __syncthreads();
    }
    if (writes && p.copies && threadIdx.x < 3) {
        const bool any = shared >= 0 && target >= 0;
        p.copies[3 * b + threadIdx.x] = threadIdx.x == 0 ? any ? shared : -1 : threadIdx.x == 1 ? any ? target : -1 : any ? held : 0;
    }
    if (shared >= 0 && target >= 0 && p.cache.k) copy_page(p.cache, p.cache, target, shared, held, part, gridDim.y);
}

__global__ __launch_bounds__(256) void kv_copy_pages_kernel(KvCache to, KvCache from, const int32_t *copies) {
    const int32_t *c = copies + 3 * (size_t)blockIdx.x;
    const int from_page = c[0], to_page = c[1], tokens = c[2];
    if (!is_page(from_page, from.pages) || !is_page(to_page, to.pages) || tokens <= 0) return;
    copy_page(to, from, to_page, from_page, tokens, blockIdx.y, gridDim.y);
}

__global__ void kv_none_missing_kernel(int32_t *missing) { *missing = 0; }

// Workgroups of a copy: until the chip is full, no more than give each 16 KB.
int copy_parts(long long copies, const KvCache &c) {
    const long long most = ((long long)c.heads * 2 * c.dim << c.page_shift) / 16384, room = 2048 / (copies < 1 ? 1 : copies), n = room < most ? room : most;
    return n < 1 ? 1 : (int)n;
}

}  // namespace

KvReservePlan plan_kv_reserve(int pages, int sequences, int width) {
    KvReservePlan r{};
    const auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    r.slices = (pages + kSlicePages - 1) / kSlicePages;
    r.words = (width + 63) / 64;
    r.slice_off = up((size_t)r.slices * (kSlicePages / 64) * 8);
    r.count_off = r.slice_off + up((size_t)r.slices * 4);
    r.shared_off = r.count_off + up((size_t)sequences * 4);
    r.lacks_off = r.shared_off + up((size_t)sequences * 4);
    r.total = r.lacks_off + up((size_t)sequences * r.words * 8);
    return r;
}

hipError_t launch_kv_release(const KvPool &pool, int32_t *table, const int32_t *first, const int32_t *last, int sequences, int width, hipStream_t stream) {
    kv_release_kernel<<<(uint32_t)(((long long)sequences * width + 255) / 256), 256, 0, stream>>>(pool, table, first, last, sequences, width);
    return hipGetLastError();
}
hipError_t launch_kv_fork(const KvForkParams &p, hipStream_t stream) {
    kv_fork_kernel<<<(uint32_t)(((long long)p.sequences * p.to_width + 255) / 256), 256, 0, stream>>>(p);
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
    kv_reserve_kernel<<<dim3(p.batch.sequences, p.cache.k ? copy_parts(p.batch.sequences, p.cache) : 1), 256, 0, stream>>>(p);
    return hipGetLastError();
}
hipError_t launch_kv_copy_pages(const KvCache &to, const KvCache &from, const int32_t *copies, int n, hipStream_t stream) {
    kv_copy_pages_kernel<<<dim3(n, copy_parts(n, to)), 256, 0, stream>>>(to, from, copies);
    return hipGetLastError();
}

}  // namespace svdq
