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

// Positions of a CTA's slice, in fours
__host__ __device__ inline int sel_slice(long long n, int slices) { return (int)(((n + slices - 1) / slices + 3) & ~3ll); }

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
constexpr uint32_t KEY_STAYS = 0xffffffffu;  // of the first and the last positions: above every score's (+inf: 0xff800000; none is 0)

__device__ __forceinline__ int2 ld_cluster(const int* p, uint32_t rank) {
    int2 v;
    asm volatile("ld.shared::cluster.v2.s32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(map_to_cta(smem_u32(p), rank)) : "memory");
    return v;
}
// The sums of p[0] and p[1] over the cluster's CTAs, each of which has them at the same place
template <int SLICES>
__device__ __forceinline__ int2 cluster_total(const int* p, int rank) {
    int2 sum = *reinterpret_cast<const int2*>(p), v[SLICES];
#pragma unroll
    for (int r = 1; r < SLICES; ++r) v[r] = ld_cluster(p, (rank + r) & (SLICES - 1));  // all under way at once
#pragma unroll
    for (int r = 1; r < SLICES; ++r) {
        sum.x += v[r].x;
        sum.y += v[r].y;
    }
    return sum;
}
// Sum of x over the lanes up to this one
__device__ __forceinline__ int scan_up(int x) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += up;
    }
    return x;
}

// A cluster takes a (chain, head), each CTA a slice of its positions, whose keys stay in shared memory, and of which a thread takes four
// neighbours at a time.  The least key that stays is found by its digits, highest first (11, 11 and 10 bits): histograms of the
// candidates that share the digits so far, and the bin in which the wanted rank falls: a warp looks for it among the sums of 32 bins
// each, then within one such group, both added up over the cluster.  Then the positions above the least key, and of those equal to it the lowest, are
// written in order: each warp has a contiguous part of the slice, whose place in the list follows from the counts of
// the parts before it.  What bounds it is the chain of these steps,
// the loads of the scores among them: 64 rows of 32K take 13.5 us on four CTAs each, 128 rows of 2K 8 us on one.  (With the bins'
// counts added up by all threads, 32 positions a warp at a time and the list written from there, 20 and 8.6.)
template <int SLICES>
__global__ void __launch_bounds__(SEL_THREADS, 2) cache_select_kernel(const EvictArgs a) {
    extern __shared__ __align__(16) uint32_t keys[];
    __shared__ __align__(8) int hist[2][SEL_BINS], group[2][SEL_BINS / 32];
    __shared__ int part[2][SEL_WARPS];
    __shared__ __align__(8) int total[2];
    __shared__ int found[3];
    const int chain = blockIdx.z, g = blockIdx.y, c = chain / a.v.L, l = chain % a.v.L, rank = (int)cluster_ctarank();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    pdl_wait();
    const int N = cache_len(a.v, c);
    int* kept = a.kept + ((size_t)chain * a.v.n_kv + g) * a.keep;
    if (a.lens_out && g == 0 && l == 0 && rank == 0 && tid == 0) a.lens_out[c] = min(N, a.keep);
    if (N <= a.keep) {  // the whole cluster
        for (int i = rank * SEL_THREADS + tid; i < a.keep; i += SLICES * SEL_THREADS) kept[i] = i < N ? i : -1;
        return;
    }
    const float* score = a.v.score + (((size_t)c * a.v.Lh + l) * a.v.n_kv + g) * a.v.cap;
    const int lo = a.n_sink, hi = N - a.n_recent;  // candidates
    const int per = sel_slice(N, SLICES), s0 = min(N, rank * per), n = min(N, s0 + per) - s0;
    auto key = [&](int i, float x) { return i >= n ? 0u : s0 + i < lo || s0 + i >= hi ? KEY_STAYS : score_key(x); };
    auto make = [&](int i) { return key(i, i < n ? score[s0 + i] : 0.f); };
    auto sync = [&]() {
        if constexpr (SLICES > 1)
            cluster_sync();
        else
            __syncthreads();
    };
    for (int i0 = tid; i0 < min((n + 3) & ~3, SEL_KEYS); i0 += 4 * SEL_THREADS) {
        float x[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) x[u] = i0 + u * SEL_THREADS < n ? score[s0 + i0 + u * SEL_THREADS] : 0.f;
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (const int i = i0 + u * SEL_THREADS; i < min((n + 3) & ~3, SEL_KEYS)) keys[i] = key(i, x[u]);
    }
    auto four = [&](int i) { return i < SEL_KEYS ? *reinterpret_cast<const uint4*>(keys + i) : make_uint4(make(i), make(i + 1), make(i + 2), make(i + 3)); };
    for (int i = tid; i < SEL_BINS; i += SEL_THREADS) hist[0][i] = 0;
    __syncthreads();
    int need = a.keep - a.n_sink - a.n_recent;  // of the candidates to keep, then of those equal to the least
    uint32_t least = need ? 0 : KEY_STAYS - 1;  // its digits so far
    int shift = 32;
    for (int pass = 0; need > 0 && shift > 0; ++pass) {
        const int bits = shift > 10 ? 11 : 10, low = shift - bits;
        int *h = hist[pass & 1], *gs = group[pass & 1];
        for (int i = 4 * tid; i < n; i += 4 * SEL_THREADS) {
            const uint4 k4 = four(i);
            const uint32_t k[4] = {k4.x, k4.y, k4.z, k4.w};
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (k[u] - 1u < KEY_STAYS - 1u && (shift == 32 || (k[u] >> shift) == least)) atomicAdd(&h[(k[u] >> low) & ((1u << bits) - 1)], 1);
        }
        __syncthreads();
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int sum = __reduce_add_sync(0xffffffffu, h[64 * warp + 32 * b + lane]);
            if (lane == 0) gs[2 * warp + b] = sum;
        }
        sync();
        for (int i = tid; i < SEL_BINS; i += SEL_THREADS) hist[(pass & 1) ^ 1][i] = 0;  // read by all before the barrier above
        if (warp == 0) {  // from the top down: which group, then which bin, a lane has two of the former, half the lanes two of the latter
            int b = 0, above = 0, count = 0;
            auto look = [&](const int* at, int n_at) {
                const int2 v = 2 * lane < n_at ? cluster_total<SLICES>(at + n_at - 2 - 2 * lane, rank) : make_int2(0, 0);
                const int upto = above + scan_up(v.x + v.y);
                const int k = __ffs(__ballot_sync(0xffffffffu, upto >= need)) - 1;
                const bool lower = __shfl_sync(0xffffffffu, upto - v.x < need, k);  // in the second of the lane's two
                count = __shfl_sync(0xffffffffu, lower ? v.x : v.y, k);
                above = __shfl_sync(0xffffffffu, lower ? upto - v.x : upto - v.x - v.y, k);
                return n_at - 1 - 2 * k - lower;
            };
            b = look(gs, SEL_BINS / 32);
            b = 32 * b + look(h + 32 * b, 32);
            if (lane == 0) {
                found[0] = b;
                found[1] = need - above;
                found[2] = count;
            }
        }
        __syncthreads();
        least = (least << bits) | (uint32_t)found[0];
        need = found[1];
        shift = low;
        if (need == found[2] && low) {  // the whole bin stays: all above the key below it
            least = (least << low) - 1;
            need = 0;
        }
    }
    const int wper = (n + 4 * SEL_THREADS - 1) / (4 * SEL_THREADS) * 128;  // positions of a warp's part
    const int w0 = warp * wper, w1 = min(n, w0 + wper);
    int over = 0, equal = 0;
    for (int i = w0 + 4 * lane; i < w1; i += 128) {
        const uint4 k = four(i);
        over += (k.x > least) + (k.y > least) + (k.z > least) + (k.w > least);
        equal += (k.x == least) + (k.y == least) + (k.z == least) + (k.w == least);
    }
    over = __reduce_add_sync(0xffffffffu, over);
    equal = __reduce_add_sync(0xffffffffu, equal);
    if (lane == 0) {
        part[0][warp] = over;
        part[1][warp] = equal;
    }
    __syncthreads();
    if (warp < 2) {
        const int sum = __reduce_add_sync(0xffffffffu, part[warp][lane]);
        if (lane == 0) total[warp] = sum;
    }
    over = __reduce_add_sync(0xffffffffu, lane < warp ? part[0][lane] : 0);
    equal = __reduce_add_sync(0xffffffffu, lane < warp ? part[1][lane] : 0);
    if constexpr (SLICES > 1) {
        cluster_sync();
        const int2 v = lane < rank ? ld_cluster(total, lane) : make_int2(0, 0);
        over += __reduce_add_sync(0xffffffffu, v.x);
        equal += __reduce_add_sync(0xffffffffu, v.y);
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    }
    // The positions of a part that stay are neighbours in the list: they go where their keys were, then out
    const int first = over + min(equal, need);
    int n_out = 0;
    for (int i = w0 + 4 * lane; i - 4 * lane < w1; i += 128) {
        const uint4 k4 = i < w1 ? four(i) : make_uint4(0, 0, 0, 0);
        const uint32_t k[4] = {k4.x, k4.y, k4.z, k4.w};
        const bool some = need && __any_sync(0xffffffffu, k[0] == least || k[1] == least || k[2] == least || k[3] == least);
        if (w1 <= SEL_KEYS && !some) {  // most of the time
            const int mine = (k[0] > least) + (k[1] > least) + (k[2] > least) + (k[3] > least), upto = scan_up(mine);
            uint32_t* to = keys + w0 + n_out + upto - mine;
            __syncwarp();
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (k[u] > least) *to++ = s0 + i + u;
            const int all = __shfl_sync(0xffffffffu, upto, 31);
            over += all;
            n_out += all;
        } else {
            int mine = 0;  // above, and equal << 16
#pragma unroll
            for (int u = 0; u < 4; ++u) mine += (k[u] > least) + ((k[u] == least) << 16);
            const int upto = scan_up(mine), ahead = upto - mine, all = __shfl_sync(0xffffffffu, upto, 31);
            int o = over + (ahead & 0xffff), e = equal + (ahead >> 16);
#pragma unroll 1
            for (int u = 0; u < 4; ++u) {
                const uint32_t ku = u == 0 ? k[0] : u == 1 ? k[1] : u == 2 ? k[2] : k[3];
                const bool up = ku > least, eq = ku == least;
                const int at = o + min(e, need);
                if (up || (eq && e < need)) {
                    if (w1 <= SEL_KEYS)
                        keys[w0 + at - first] = s0 + i + u;
                    else if (at < a.keep)
                        kept[at] = s0 + i + u;
                }
                o += up;
                e += eq;
            }
            over += all & 0xffff;
            equal += all >> 16;
            if (w1 <= SEL_KEYS) n_out = over + min(equal, need) - first;
        }
        __syncwarp();
    }
    for (int i = lane; i < n_out; i += 32)
        if (first + i < a.keep) kept[first + i] = keys[w0 + i];
    if constexpr (SLICES > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");  // no CTA leaves while another reads its shared memory
}

template <int SLICES>
cudaError_t select(const EvictArgs& a, cudaStream_t st) {
    static PerDevice<SmemOptIn> once;
    constexpr size_t smem = SEL_KEYS * sizeof(uint32_t);
    cudaError_t e = smem_opt_in(reinterpret_cast<const void*>(cache_select_kernel<SLICES>), smem, once);
    if (e != cudaSuccess) return e;
    return launch_kernel(cache_select_kernel<SLICES>, dim3(SLICES, a.v.n_kv, a.v.n_ctx * a.v.L), dim3(SEL_THREADS),
                         std::min<size_t>(smem, sel_slice(a.v.cap, SLICES) * sizeof(uint32_t)), st, true, SLICES, a);
}

// ---------------------------------------------------------------- eviction: their rows
constexpr int CM_SLOTS = 8, CM_WAY = 2;

// A warp takes CM_SLOTS survivors: a lane looks up where one comes from and goes to, then all move units of their key and value
// rows, CM_WAY under way in each lane.  Bound by HBM, whose reads come row by row: 203 MB in rows of 256 bytes, read and written, take
// 65 us, 6.2 TB/s, 128 x 1024 rows of 2 x 128 bytes 13 us.  (The two with their select: 2 under way 88.7 and 14.5 us, 4 under way
// 99.6 and 16.1, 8 under way 121 and 19.6: few loads a warp and many warps.)
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
        if (from >= 0) {  // (past the survivors, an entry of the target's table need not name a page)
            const int p1 = cache_page(a.v, a.to + (size_t)c * a.to_width, i >> a.v.page_log2);
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
    // A row over as many CTAs of a cluster as the SMs hold, two each, and slices of SEL_SLICE positions of what the table covers (the
    // lengths are on the device).  (128 rows of 2K take
    // 14.1 us with their compaction on one CTA each, 17.8 on two; 64 rows of 32K 99, 84, 80 and 82 on one, two, four and eight; 8
    // rows of 120000 202 on one and 98 on eight.)
    const long long rows = (long long)v.n_ctx * v.L * v.n_kv;
    int slices = 1;
    while (slices < 8 && 2 * slices * rows <= 2 * s.sms && v.cap / (2 * slices) >= SEL_SLICE) slices *= 2;
    cudaError_t e = slices == 1 ? select<1>(a, st) : slices == 2 ? select<2>(a, st) : slices == 4 ? select<4>(a, st) : select<8>(a, st);
    if (e != cudaSuccess) return e;
    if (!cache_vec(v, el)) return s.dtype == 0 ? compact<uint32_t>(a, st) : compact<uint16_t>(a, st);
    in_units(a.v, 16 / el);
    a.units = s.hd * el / 16;
    return compact<uint4>(a, st);
}

}  // namespace mone
