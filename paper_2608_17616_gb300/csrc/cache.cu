// The paged cache's data movers: appending new tokens (mone_cache_append) and cutting a cache down to its first positions,
// its last and the best scored others (mone_cache_evict).  Rows are moved in units of 16 bytes, or of one element where
// some row does not start on a 16-byte boundary.
#include <algorithm>

#include "cache_common.cuh"
#include "per_device.h"

namespace mone {

namespace {

constexpr int CP_THREADS = 256;

// ---------------------------------------------------------------- append
struct AppendArgs {
    CacheView v;
    const void *K, *V;               // element strides s0 (context), s1 (layer), s2 (head), s3 (token), in units
    long long s0, s1, s2, s3;
    int n_tok, units;                // units of a row
    const int* counts;
    int* lens_out;
};

// A thread moves one unit of a token's key row and one of its value row.  Bound by HBM; one token a context by
// the launch and two dependent loads (length, page) ahead of the copy.
template <typename U>
__global__ void __launch_bounds__(CP_THREADS) cache_append_kernel(const AppendArgs a) {
    const int chain = blockIdx.z, g = blockIdx.y, c = chain / a.v.L, l = chain % a.v.L;
    pdl_wait();
    pdl_trigger();
    const int len = cache_len(a.v, c);
    const int n = a.counts ? min(max(a.counts[c], 0), a.n_tok) : a.n_tok;
    if (a.lens_out && blockIdx.x == 0 && g == 0 && l == 0 && threadIdx.x == 0)
        a.lens_out[c] = (int)min((long long)len + n, a.v.cap);
    const long long e = (long long)blockIdx.x * CP_THREADS + threadIdx.x;
    const int i = (int)(e / a.units), u = (int)(e % a.units);
    if (i >= n) return;
    const long long pos = (long long)len + i;
    if (pos >= a.v.cap) {
        cache_fail(a.v.status, DS_CACHE_LEN);
        return;
    }
    if (u == 0 && a.v.score) a.v.score[(((size_t)c * a.v.Lh + l) * a.v.n_kv + g) * a.v.cap + pos] = 0.f;
    const int page = cache_page(a.v, a.v.table + (size_t)c * a.v.width, (int)(pos >> a.v.page_log2));
    if (page < 0) return;
    const long long src = c * a.s0 + l * a.s1 + g * a.s2 + i * a.s3 + u;
    const long long dst = l * a.v.s_layer + page * a.v.s_page + g * a.v.s_head + (pos & ((1 << a.v.page_log2) - 1)) * a.v.s_pos + u;
    const U k = static_cast<const U*>(a.K)[src], v = static_cast<const U*>(a.V)[src];
    static_cast<U*>(a.v.K)[dst] = k;
    static_cast<U*>(a.v.V)[dst] = v;
}

// The strides of v in units of `per` elements.
void in_units(CacheView& v, int per) {
    v.s_layer /= per;
    v.s_page /= per;
    v.s_head /= per;
    v.s_pos /= per;
}

template <typename U>
cudaError_t append(AppendArgs a, cudaStream_t st) {
    const dim3 grid((unsigned)(((long long)a.n_tok * a.units + CP_THREADS - 1) / CP_THREADS), a.v.n_kv, a.v.n_ctx * a.v.L);
    return launch_kernel(cache_append_kernel<U>, grid, dim3(CP_THREADS), 0, st, true, 1, a);
}

// ---------------------------------------------------------------- eviction: which positions stay
constexpr int SEL_THREADS = 1024, SEL_WARPS = SEL_THREADS / 32, SEL_BINS = 2048;
constexpr int SEL_KEYS = 16384;  // keys that a CTA keeps on chip; of a longer slice it reads the others' scores again in each pass
constexpr int SEL_SLICE = 2048;  // positions of a CTA's slice at least, where a row is split

struct EvictArgs {
    CacheView v;
    int keep, n_sink, n_recent, units;
    const int* to;
    int to_width;
    long long to_cap;
    float* to_score;
    int* kept;       // [n_ctx * L][n_kv][keep]
    int* lens_out;
};

// Scores as unsigned numbers of the same order: NaN as -inf, -0 as 0.
__device__ __forceinline__ uint32_t score_key(float f) {
    f = isnan(f) ? -INFINITY : f + 0.f;
    const uint32_t u = __float_as_uint(f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
constexpr uint32_t KEY_STAYS = 0xffffffffu;  // of the first and the last positions: above every score's (+inf: 0xff800000)

// int of CTA `rank` of the cluster at the place of `p` in this one
__device__ __forceinline__ int ld_cluster(const int* p, uint32_t rank) {
    int v;
    asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(map_to_cta(smem_u32(p), rank)) : "memory");
    return v;
}

// A cluster takes a (chain, head), each CTA a slice of its positions, whose keys stay in shared memory.  The least key that
// stays is found by its digits, highest first (11, 11 and 10 bits): histograms of the candidates that share the digits so
// far, added up over the cluster, and the bin in which the wanted rank falls.  Then the positions above it, and of those equal
// to it the lowest, are written in order: each warp has a contiguous part of the slice, whose place in the list follows from
// the counts of the parts before it.  What bounds it is the chain of passes, each a shared-memory histogram, a cluster barrier and a scan:
// 64 rows of up to 32K take 13 us (one CTA a row, scores read again in each pass: 37).
__global__ void __launch_bounds__(SEL_THREADS) cache_select_kernel(const EvictArgs a, int slices) {
    extern __shared__ uint32_t keys[];
    __shared__ int hist[2][SEL_BINS];
    __shared__ int part[2][SEL_WARPS], total[2];
    __shared__ int found[2];
    const int chain = blockIdx.z, g = blockIdx.y, c = chain / a.v.L, l = chain % a.v.L, rank = (int)cluster_ctarank();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    pdl_wait();
    pdl_trigger();
    const int N = cache_len(a.v, c);
    int* kept = a.kept + ((size_t)chain * a.v.n_kv + g) * a.keep;
    if (a.lens_out && g == 0 && l == 0 && rank == 0 && tid == 0) a.lens_out[c] = min(N, a.keep);
    if (N <= a.keep) {  // the whole cluster
        for (int i = rank * SEL_THREADS + tid; i < a.keep; i += slices * SEL_THREADS) kept[i] = i < N ? i : -1;
        return;
    }
    const float* score = a.v.score + (((size_t)c * a.v.Lh + l) * a.v.n_kv + g) * a.v.cap;
    const int lo = a.n_sink, hi = N - a.n_recent;  // candidates
    const int per = (N + slices - 1) / slices, s0 = min(N, rank * per), n = min(N, s0 + per) - s0;
    auto make = [&](int i) { return s0 + i < lo || s0 + i >= hi ? KEY_STAYS : score_key(score[s0 + i]); };
    for (int i = tid; i < min(n, SEL_KEYS); i += SEL_THREADS) keys[i] = make(i);
    auto key = [&](int i) { return i < SEL_KEYS ? keys[i] : make(i); };
    for (int i = tid; i < SEL_BINS; i += SEL_THREADS) hist[0][i] = 0;
    __syncthreads();
    int need = a.keep - a.n_sink - a.n_recent;  // of the candidates to keep, then of those equal to the least
    uint32_t prefix = need ? 0 : KEY_STAYS - 1;
    int shift = 32, pass = 0;
    while (need > 0 && shift > 0) {
        const int bits = shift > 10 ? 11 : 10, low = shift - bits;
        int* h = hist[pass & 1];
        for (int i = tid; i < n; i += SEL_THREADS) {
            const uint32_t k = key(i);
            if (k != KEY_STAYS && (shift == 32 || (k >> shift) == prefix)) atomicAdd(&h[(k >> low) & ((1u << bits) - 1)], 1);
        }
        if (slices > 1)
            cluster_sync();
        else
            __syncthreads();
        for (int i = tid; i < SEL_BINS; i += SEL_THREADS) hist[(pass & 1) ^ 1][i] = 0;  // read by all before the barrier above
        // candidates in the bins from a thread's pair up, counted from the top
        const int b1 = SEL_BINS - 1 - 2 * tid;
        int h1 = h[b1], h0 = h[b1 - 1];
        for (int r = 1; r < slices; ++r) {
            const int other = rank + r < slices ? rank + r : rank + r - slices;
            h1 += ld_cluster(h + b1, other);
            h0 += ld_cluster(h + b1 - 1, other);
        }
        int sum = h1 + h0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int up = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += up;
        }
        if (lane == 31) part[0][warp] = sum;
        __syncthreads();
        const int mine = part[0][lane];
        const int above = __reduce_add_sync(0xffffffffu, lane < warp ? mine : 0) + sum - h1 - h0;  // in the bins over the pair
        if (above < need && need <= above + h1) {
            found[0] = b1;
            found[1] = need - above;
        } else if (above + h1 < need && need <= above + h1 + h0) {
            found[0] = b1 - 1;
            found[1] = need - above - h1;
        }
        __syncthreads();
        prefix = (prefix << bits) | (uint32_t)found[0];
        need = found[1];
        shift = low;
        ++pass;
    }
    const int wper = (n + SEL_THREADS - 1) / SEL_THREADS * 32;  // positions of a warp's part
    const int w0 = warp * wper, w1 = min(n, w0 + wper);
    int over = 0, equal = 0;
    for (int i = w0 + lane; i - lane < w1; i += 32) {
        const uint32_t k = i < w1 ? key(i) : 0;
        over += __popc(__ballot_sync(0xffffffffu, i < w1 && k > prefix));
        equal += __popc(__ballot_sync(0xffffffffu, i < w1 && k == prefix));
    }
    if (lane == 0) {
        part[0][warp] = over;
        part[1][warp] = equal;
    }
    __syncthreads();
    if (warp < 2) {
        const int sum = __reduce_add_sync(0xffffffffu, part[warp][lane]);
        if (lane == 0) total[warp] = sum;
    }
    if (slices > 1)
        cluster_sync();
    else
        __syncthreads();
    over = __reduce_add_sync(0xffffffffu, lane < warp ? part[0][lane] : 0);
    equal = __reduce_add_sync(0xffffffffu, lane < warp ? part[1][lane] : 0);
    if (slices > 1) {
        over += __reduce_add_sync(0xffffffffu, lane < rank ? ld_cluster(total, lane) : 0);
        equal += __reduce_add_sync(0xffffffffu, lane < rank ? ld_cluster(total + 1, lane) : 0);
        cluster_sync();  // no CTA leaves while another reads its shared memory
    }
    for (int i = w0 + lane; i - lane < w1; i += 32) {
        const uint32_t k = i < w1 ? key(i) : 0;
        const bool up = i < w1 && k > prefix, eq = i < w1 && k == prefix;
        const uint32_t ups = __ballot_sync(0xffffffffu, up), eqs = __ballot_sync(0xffffffffu, eq), below = (1u << lane) - 1;
        const int e = equal + __popc(eqs & below), at = over + __popc(ups & below) + min(e, need);
        if ((up || (eq && e < need)) && at < a.keep) kept[at] = s0 + i;
        over += __popc(ups);
        equal += __popc(eqs);
    }
}

// ---------------------------------------------------------------- eviction: their rows
constexpr int CM_SLOTS = 8, CM_WAY = 2;

// A warp takes CM_SLOTS survivors: a lane looks up where one comes from and goes to, then all move units of their key and value
// rows, CM_WAY under way in each lane.
template <typename U>
__global__ void __launch_bounds__(CP_THREADS) cache_compact_kernel(const EvictArgs a) {
    const int chain = blockIdx.z, g = blockIdx.y, c = chain / a.v.L, l = chain % a.v.L, lane = threadIdx.x & 31;
    const int i0 = (blockIdx.x * (CP_THREADS / 32) + (threadIdx.x >> 5)) * CM_SLOTS;
    pdl_wait();
    if (i0 >= a.keep) return;
    long long src = -1, dst = -1;
    const int i = i0 + lane;
    if (lane < CM_SLOTS && i < a.keep) {
        const int mask = (1 << a.v.page_log2) - 1, from = a.kept[((size_t)chain * a.v.n_kv + g) * a.keep + i];
        const int p1 = cache_page(a.v, a.to + (size_t)c * a.to_width, i >> a.v.page_log2);
        if (from >= 0) {
            const size_t row = ((size_t)c * a.v.Lh + l) * a.v.n_kv + g;
            const int p0 = cache_page(a.v, a.v.table + (size_t)c * a.v.width, from >> a.v.page_log2);
            a.to_score[row * a.to_cap + i] = a.v.score[row * a.v.cap + from];
            if (p0 >= 0 && p1 >= 0) {
                const long long base = l * a.v.s_layer + g * a.v.s_head;
                src = base + p0 * a.v.s_page + (from & mask) * a.v.s_pos;
                dst = base + p1 * a.v.s_page + (i & mask) * a.v.s_pos;
            }
        }
    }
    // units of a slot: of its key row, then of its value row (a power of two each)
    const int unit_log2 = 31 - __clz(a.units);
    U* const pool[2] = {static_cast<U*>(a.v.K), static_cast<U*>(a.v.V)};
    for (int e0 = lane; e0 < CM_SLOTS << (unit_log2 + 1); e0 += CM_WAY * 32) {
        U x[CM_WAY];
        U* to[CM_WAY];
#pragma unroll
        for (int k = 0; k < CM_WAY; ++k) {
            const int e = e0 + k * 32, slot = e >> (unit_log2 + 1), o = e & (a.units - 1);
            const long long s = __shfl_sync(0xffffffffu, src, slot), d = __shfl_sync(0xffffffffu, dst, slot);
            U* const p = (e >> unit_log2) & 1 ? pool[1] : pool[0];
            to[k] = nullptr;
            if (s >= 0 && slot < CM_SLOTS) {
                x[k] = p[s + o];
                to[k] = p + d + o;
            }
        }
#pragma unroll
        for (int k = 0; k < CM_WAY; ++k)
            if (to[k]) *to[k] = x[k];
    }
}

template <typename U>
cudaError_t compact(const EvictArgs& a, cudaStream_t st) {
    const int slots = CM_SLOTS * CP_THREADS / 32;
    const dim3 grid((unsigned)((a.keep + slots - 1) / slots), a.v.n_kv, a.v.n_ctx * a.v.L);
    return launch_kernel(cache_compact_kernel<U>, grid, dim3(CP_THREADS), 0, st, true, 1, a);
}

}  // namespace

cudaError_t launch_cache_append(const DevState& s, const CacheView& v, const void* K, const void* V, const long long* strides,
                                int n_tok, const int* counts, int* lens_out, cudaStream_t st) {
    const int el = s.dtype == 0 ? 4 : 2;
    AppendArgs a{v, K, V, strides[0], strides[1], strides[2], strides[3], n_tok, s.hd, counts, lens_out};
    const bool vec = cache_vec(v, el) && (((uintptr_t)K | (uintptr_t)V) & 15u) == 0 && a.s0 * el % 16 == 0 && a.s1 * el % 16 == 0 &&
                     a.s2 * el % 16 == 0 && a.s3 * el % 16 == 0;
    if (!vec) return s.dtype == 0 ? append<uint32_t>(a, st) : append<uint16_t>(a, st);
    const int per = 16 / el;
    in_units(a.v, per);
    a.s0 /= per; a.s1 /= per; a.s2 /= per; a.s3 /= per;
    a.units = s.hd / per;
    return append<uint4>(a, st);
}

cudaError_t launch_cache_evict(const DevState& s, const CacheView& v, int keep, int n_sink, int n_recent, const int* to, int to_width,
                               float* to_score, int* kept, int* lens_out, cudaStream_t st) {
    const int el = s.dtype == 0 ? 4 : 2;
    EvictArgs a{v, keep, n_sink, n_recent, s.hd, to, to_width, (long long)to_width << v.page_log2, to_score, kept, lens_out};
    // A row over as many CTAs of a cluster as the SMs hold, two each, and slices of SEL_SLICE positions.  (8 rows of 2K take 8.5 us
    // with their compaction on one CTA each, 11.0 on two; 64 rows of up to 32K 88.7 on two, 85.4 on four, 126 on eight.)
    const long long rows = (long long)v.n_ctx * v.L * v.n_kv;
    int slices = 1;
    while (slices < 8 && 2 * slices * rows <= 2 * s.sms && v.cap / (2 * slices) >= SEL_SLICE) slices *= 2;
    static PerDevice<SmemOptIn> once;
    constexpr size_t smem = SEL_KEYS * sizeof(uint32_t);
    cudaError_t e = smem_opt_in(reinterpret_cast<const void*>(cache_select_kernel), smem, once);
    if (e != cudaSuccess) return e;
    e = launch_kernel(cache_select_kernel, dim3(slices, v.n_kv, v.n_ctx * v.L), dim3(SEL_THREADS),
                      std::min<size_t>(smem, (v.cap + slices - 1) / slices * sizeof(uint32_t)), st, true, slices, a, slices);
    if (e != cudaSuccess) return e;
    if (!cache_vec(v, el)) return s.dtype == 0 ? compact<uint32_t>(a, st) : compact<uint16_t>(a, st);
    in_units(a.v, 16 / el);
    a.units = s.hd * el / 16;
    return compact<uint4>(a, st);
}

}  // namespace mone
