// Pages of the paged caches: taken from the list of free ones for new tokens, with the tokens' slots (mone_cache_reserve), and given back
// (mone_cache_release).
//
// Each CTA adds up what the contexts before its own take or give, so nothing is passed between CTAs: the list's new length goes to another
// word than the old one, which all read.
#include <algorithm>
#include <climits>

#include "cache_common.cuh"

namespace mone {

namespace {

constexpr int PG_THREADS = 256, PG_WARPS = PG_THREADS / 32;
constexpr int PG_EACH = 4;  // tokens or pages of a thread

struct PagesArgs {
    PagesView v;
    int n_tok;
    const int* counts;   // reserve: tokens of each context; release: positions that it keeps
    int* granted;
    long long* slots;
    int *lens_out, *n_free_out;
};

__device__ __forceinline__ int pages_len(const PagesView& v, int c) {
    const int n = v.lens[c];
    if (n < 0 || n > v.cap) {
        cache_fail(v.status, DS_CACHE_LEN);
        return n < 0 ? 0 : (int)v.cap;
    }
    return n;
}
__device__ __forceinline__ int pages_free(const PagesView& v) {
    const int n = *v.n_free;
    if (n < 0 || n > v.n_pages) {
        cache_fail(v.status, DS_CACHE_FREE);
        return n < 0 ? 0 : v.n_pages;
    }
    return n;
}
__device__ __forceinline__ int pages_of(const PagesView& v, long long positions) { return (int)((positions + (1 << v.page_log2) - 1) >> v.page_log2); }

// Inclusive sum over the block's threads; `total` the last one's
__device__ __forceinline__ long long block_scan(long long x, long long& total) {
    __shared__ long long part[PG_WARPS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long up = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += up;
    }
    __syncthreads();
    if (lane == 31) part[warp] = x;
    __syncthreads();
    total = 0;
#pragma unroll
    for (int w = 0; w < PG_WARPS; ++w) {
        if (w == warp) x += total;
        total += part[w];
    }
    return x;
}

// The context's place among all: pages of those before it and its own (asked), and of all that are there (taken: the largest sum that
// is at most `limit`).
struct PagesPlace {
    long long before;
    int mine;
    long long taken;
};
template <typename F>
__device__ __forceinline__ PagesPlace place_of(const PagesView& v, int c, long long limit, F need) {
    __shared__ long long found_before, found_taken;
    __shared__ int found_mine;
    if (threadIdx.x == 0) found_taken = 0;
    long long sum = 0;
    for (int c0 = 0; c0 < v.n_ctx; c0 += PG_THREADS) {
        const int k = c0 + threadIdx.x, n = k < v.n_ctx ? need(k) : 0;
        long long total;
        const long long upto = sum + block_scan(n, total);
        if (k == c) {
            found_before = upto - n;
            found_mine = n;
        }
        // sums only grow: the last that fits is the largest
        const bool fits = upto <= limit;
        long long best = fits ? upto : 0;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            const long long x = __shfl_xor_sync(0xffffffffu, best, o);
            best = x > best ? x : best;
        }
        if ((threadIdx.x & 31) == 0 && best) atomicMax(&found_taken, best);
        sum += total;
    }
    __syncthreads();
    return {found_before, found_mine, found_taken};
}

// Bound by its launch and three dependent loads (lengths, the list, slots) where few tokens come; by the slots' 8 bytes a token for
// prompts.
__global__ void __launch_bounds__(PG_THREADS) cache_reserve_kernel(const PagesArgs a) {
    const PagesView& v = a.v;
    const int c = blockIdx.y, page_size = 1 << v.page_log2;
    pdl_wait();
    const int n_free = pages_free(v);
    auto count_of = [&](int k) { return a.counts ? min(max(a.counts[k], 0), a.n_tok) : a.n_tok; };
    const PagesPlace p = place_of(v, c, n_free, [&](int k) {
        const long long len = pages_len(v, k), end = len + count_of(k);
        return end > v.cap ? 0 : pages_of(v, end) - pages_of(v, len);
    });
    const int len = pages_len(v, c), held = pages_of(v, len);
    int count = count_of(c);
    if ((long long)len + count > v.cap || (p.mine && p.before + p.mine > n_free)) count = 0;
    const int mine = count ? p.mine : 0;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        if (a.granted) a.granted[c] = count;
        if (a.lens_out) a.lens_out[c] = len + count;
        if (c == 0) *a.n_free_out = n_free - (int)p.taken;
    }
    int* table = v.table + (size_t)c * v.width;
    const int* fresh = v.free + (n_free - p.taken + p.before);  // its new pages
    auto page_at = [&](int k) {
        const int page = fresh[k];
        if ((unsigned)page < (unsigned)v.n_pages) return page;
        cache_fail(v.status, DS_CACHE_PAGE);
        return -1;
    };
    const int stride = gridDim.x * PG_THREADS, first = blockIdx.x * PG_THREADS + threadIdx.x;
    for (int k = first; k < mine; k += stride) table[held + k] = page_at(k);
    if (!a.slots) return;
    long long* slots = a.slots + (size_t)c * a.n_tok;
    for (int i = first; i < a.n_tok; i += stride) {
        long long slot = -1;
        if (i < count) {
            const int pos = len + i, block = pos >> v.page_log2;
            const int page = block < held ? table[block] : page_at(block - held);
            if ((unsigned)page < (unsigned)v.n_pages)
                slot = (long long)page << v.page_log2 | (pos & (page_size - 1));
            else
                cache_fail(v.status, DS_CACHE_PAGE);
        }
        slots[i] = slot;
    }
}

__global__ void __launch_bounds__(PG_THREADS) cache_release_kernel(const PagesArgs a) {
    const PagesView& v = a.v;
    const int c = blockIdx.y;
    pdl_wait();
    const int n_free = pages_free(v);
    auto stay_of = [&](int k, int len) { return a.counts ? min(max(a.counts[k], 0), len) : 0; };
    const PagesPlace p = place_of(v, c, LLONG_MAX, [&](int k) {
        const int len = pages_len(v, k);
        return pages_of(v, len) - pages_of(v, stay_of(k, len));
    });
    const int len = pages_len(v, c), stay = stay_of(c, len), first_page = pages_of(v, stay);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        if (a.lens_out) a.lens_out[c] = stay;
        if (c == 0) {
            if (n_free + p.taken > v.n_pages) cache_fail(v.status, DS_CACHE_FREE);  // more than there are
            *a.n_free_out = (int)min(n_free + p.taken, (long long)v.n_pages);
        }
    }
    int* table = v.table + (size_t)c * v.width + first_page;
    for (int k = blockIdx.x * PG_THREADS + threadIdx.x; k < p.mine; k += gridDim.x * PG_THREADS) {
        const int page = table[k];
        const long long at = n_free + p.before + k;
        if ((unsigned)page >= (unsigned)v.n_pages) cache_fail(v.status, DS_CACHE_PAGE);
        if (at < v.n_pages) v.free[at] = page;
        table[k] = -1;
    }
}

// CTAs of a context, for n items at most
unsigned ctas_for(long long n) { return (unsigned)std::min<long long>(std::max<long long>((n + PG_THREADS * PG_EACH - 1) / (PG_THREADS * PG_EACH), 1), 1024); }

}  // namespace

cudaError_t launch_cache_reserve(const PagesView& v, int n_tok, const int* counts, int* granted, long long* slots, int* lens_out, int* n_free_out,
                                 cudaStream_t st) {
    const PagesArgs a{v, n_tok, counts, granted, slots, lens_out, n_free_out};
    const dim3 grid(ctas_for(slots ? n_tok : (n_tok >> v.page_log2) + 1), v.n_ctx);
    return launch_kernel(cache_reserve_kernel, grid, dim3(PG_THREADS), 0, st, true, 1, a);
}

cudaError_t launch_cache_release(const PagesView& v, const int* keep, int* lens_out, int* n_free_out, cudaStream_t st) {
    const PagesArgs a{v, 0, keep, nullptr, nullptr, lens_out, n_free_out};
    return launch_kernel(cache_release_kernel, dim3(ctas_for(v.width), v.n_ctx), dim3(PG_THREADS), 0, st, true, 1, a);
}

}  // namespace mone
