// The paged cache's data movers: appending new tokens (mone_cache_append) and cutting a cache down to its first positions,
// its last and the best scored others (mone_cache_evict).  Rows are moved in units of 16 bytes, or of one element where
// some row does not start on a 16-byte boundary.
#include <algorithm>

#include "cache_common.cuh"

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
    const int len = cache_len(a.v, c);
    const int n = a.counts ? min(max(__ldg(a.counts + c), 0), a.n_tok) : a.n_tok;
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
    cache_append_kernel<U><<<grid, CP_THREADS, 0, st>>>(a);
    return cudaGetLastError();
}

// ---------------------------------------------------------------- eviction: which positions stay
constexpr int SEL_THREADS = 1024, SEL_BINS = 2048;

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

// One CTA per (chain, head).  The least key that stays is found by its digits, highest first (11, 11 and 10 bits: a
// histogram of the candidates that share the digits so far, and the bin in which the wanted rank falls), then the
// positions above it, and of those equal to it the lowest, are written in order: each warp takes a contiguous part,
// whose place in the list follows from the parts' counts.
__global__ void __launch_bounds__(SEL_THREADS) cache_select_kernel(const EvictArgs a) {
    __shared__ int hist[SEL_BINS];
    __shared__ int part[2][SEL_THREADS / 32];
    __shared__ int found[2];
    const int chain = blockIdx.y, g = blockIdx.x, c = chain / a.v.L, l = chain % a.v.L;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int N = cache_len(a.v, c);
    int* kept = a.kept + ((size_t)chain * a.v.n_kv + g) * a.keep;
    if (a.lens_out && g == 0 && l == 0 && tid == 0) a.lens_out[c] = min(N, a.keep);
    if (N <= a.keep) {
        for (int i = tid; i < a.keep; i += SEL_THREADS) kept[i] = i < N ? i : -1;
        return;
    }
    const float* score = a.v.score + (((size_t)c * a.v.Lh + l) * a.v.n_kv + g) * a.v.cap;
    const int lo = a.n_sink, hi = N - a.n_recent;  // candidates
    int need = a.keep - a.n_sink - a.n_recent;     // of them to keep, then of those equal to the least
    uint32_t prefix = 0;
    int shift = 32;
    if (need == 0) prefix = 0xffffffffu;  // above every key
    while (need > 0 && shift > 0) {
        const int bits = shift > 10 ? 11 : 10;
        for (int i = tid; i < SEL_BINS; i += SEL_THREADS) hist[i] = 0;
        __syncthreads();
        const int low = shift - bits;
        for (int i = lo + tid; i < hi; i += SEL_THREADS) {
            const uint32_t k = score_key(score[i]);
            if (shift == 32 || (k >> shift) == prefix) atomicAdd(&hist[(k >> low) & ((1u << bits) - 1)], 1);
        }
        __syncthreads();
        // candidates in the bins from a thread's pair up, counted from the top
        const int b1 = SEL_BINS - 1 - 2 * tid, h1 = hist[b1], h0 = hist[b1 - 1];
        int sum = h1 + h0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int up = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += up;
        }
        if (lane == 31) part[0][warp] = sum;
        __syncthreads();
        int before = 0;
        for (int w = 0; w < warp; ++w) before += part[0][w];
        const int above = before + sum - h1 - h0;  // in the bins over the pair
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
    }
    const int per = (N + SEL_THREADS - 1) / SEL_THREADS * 32;  // positions of a warp's part
    const int p0 = warp * per, p1 = min(N, p0 + per);
    int over = 0, equal = 0;
    for (int p = p0 + lane; p - lane < p1; p += 32) {
        const bool forced = p < p1 && (p < lo || p >= hi);
        const uint32_t k = p < p1 && !forced ? score_key(score[p]) : 0;
        over += __popc(__ballot_sync(0xffffffffu, forced || k > prefix));
        equal += __popc(__ballot_sync(0xffffffffu, !forced && p < p1 && k == prefix));
    }
    if (lane == 0) {
        part[0][warp] = over;
        part[1][warp] = equal;
    }
    __syncthreads();
    over = equal = 0;
    for (int w = 0; w < warp; ++w) {
        over += part[0][w];
        equal += part[1][w];
    }
    for (int p = p0 + lane; p - lane < p1; p += 32) {
        const bool forced = p < p1 && (p < lo || p >= hi);
        const uint32_t k = p < p1 && !forced ? score_key(score[p]) : 0;
        const bool up = forced || k > prefix, eq = !forced && p < p1 && k == prefix;
        const uint32_t ups = __ballot_sync(0xffffffffu, up), eqs = __ballot_sync(0xffffffffu, eq), below = (1u << lane) - 1;
        const int e = equal + __popc(eqs & below), at = over + __popc(ups & below) + min(e, need);
        if ((up || (eq && e < need)) && at < a.keep) kept[at] = p;
        over += __popc(ups);
        equal += __popc(eqs);
    }
}

// ---------------------------------------------------------------- eviction: their rows
// A thread moves one unit of a survivor's key row and one of its value row.
template <typename U>
__global__ void __launch_bounds__(CP_THREADS) cache_compact_kernel(const EvictArgs a) {
    const int chain = blockIdx.z, g = blockIdx.y, c = chain / a.v.L, l = chain % a.v.L;
    const long long e = (long long)blockIdx.x * CP_THREADS + threadIdx.x;
    const int i = (int)(e / a.units), u = (int)(e % a.units);
    if (i >= a.keep) return;
    const int from = a.kept[((size_t)chain * a.v.n_kv + g) * a.keep + i];
    if (from < 0) return;
    const size_t row = ((size_t)c * a.v.Lh + l) * a.v.n_kv + g;
    if (u == 0) a.to_score[row * a.to_cap + i] = a.v.score[row * a.v.cap + from];
    const int mask = (1 << a.v.page_log2) - 1;
    const int p0 = cache_page(a.v, a.v.table + (size_t)c * a.v.width, from >> a.v.page_log2);
    const int p1 = cache_page(a.v, a.to + (size_t)c * a.to_width, i >> a.v.page_log2);
    if (p0 < 0 || p1 < 0) return;
    const long long base = l * a.v.s_layer + g * a.v.s_head + u;
    const long long src = base + p0 * a.v.s_page + (from & mask) * a.v.s_pos, dst = base + p1 * a.v.s_page + (i & mask) * a.v.s_pos;
    const U k = static_cast<const U*>(a.v.K)[src], v = static_cast<const U*>(a.v.V)[src];
    static_cast<U*>(a.v.K)[dst] = k;
    static_cast<U*>(a.v.V)[dst] = v;
}

template <typename U>
cudaError_t compact(const EvictArgs& a, cudaStream_t st) {
    const dim3 grid((unsigned)(((long long)a.keep * a.units + CP_THREADS - 1) / CP_THREADS), a.v.n_kv, a.v.n_ctx * a.v.L);
    cache_compact_kernel<U><<<grid, CP_THREADS, 0, st>>>(a);
    return cudaGetLastError();
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
    cache_select_kernel<<<dim3(v.n_kv, v.n_ctx * v.L), SEL_THREADS, 0, st>>>(a);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    if (!cache_vec(v, el)) return s.dtype == 0 ? compact<uint32_t>(a, st) : compact<uint16_t>(a, st);
    in_units(a.v, 16 / el);
    a.units = s.hd * el / 16;
    return compact<uint4>(a, st);
}

}  // namespace mone
