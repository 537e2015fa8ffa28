// The 4-bit paged cache's data movers: appending new tokens (mone_cache4_append), a context's positions as dense keys and
// values (mone_cache4_read), and the rows of an eviction (mone_cache4_evict).
#include <algorithm>

#include "cache4_common.cuh"
#include "per_device.h"

namespace mone {

namespace {

constexpr int C4_THREADS = 256;

// A layer's KV head in the pools
struct FourRows {
    uint8_t *K, *V, *Ks, *Vs;
    long long s_page, s_pos, c_page, c_pos;
    int mask;
    __device__ FourRows(const Cache4View& f, int l, int g)
        : s_page(f.v.s_page), s_pos(f.v.s_pos), c_page(f.c_page), c_pos(f.c_pos), mask((1 << f.v.page_log2) - 1) {
        const long long code = l * f.v.s_layer + g * f.v.s_head, scale = l * f.c_layer + g * f.c_head;
        K = static_cast<uint8_t*>(f.v.K) + code;
        V = static_cast<uint8_t*>(f.v.V) + code;
        Ks = f.Ks + scale;
        Vs = f.Vs + scale;
    }
    __device__ long long code(int page, int pos) const { return page * s_page + (pos & mask) * s_pos; }
    __device__ long long scale(int page, int pos) const { return page * c_page + (pos & mask) * c_pos; }
};

// ---------------------------------------------------------------- append
struct Append4Args {
    Cache4View f;
    const void *K, *V;
    long long s0, s1, s2, s3;  // element strides (context, layer, head, token)
    int n_tok, groups;         // of a row
    float k_inv, v_inv;        // 2^-exp
    const int* counts;
    int* lens_out;
};

// 16 neighbours
template <typename T, bool VEC>
__device__ __forceinline__ void load16(const T* p, float (&x)[16]) {
    if constexpr (VEC) {
        constexpr int PER = 16 / sizeof(T);
        uint4 u[16 / PER];
#pragma unroll
        for (int i = 0; i < 16 / PER; ++i) u[i] = reinterpret_cast<const uint4*>(p)[i];
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = to_f<T>(reinterpret_cast<const T*>(&u[i / PER])[i % PER]);
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = to_f<T>(p[i]);
    }
}

// A group's 16 codes (two words) and its scale
__device__ __forceinline__ uint32_t encode16(const float (&x)[16], float unit_inv, uint2& codes) {
    float most = 0.f;
    bool nan = false;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        most = fmaxf(most, fabsf(x[i]));
        nan |= isnan(x[i]);
    }
    const uint32_t scale = nan ? 0x7fu : encode_scale(most * unit_inv);
    const float s = scale_float(scale), inv = __frcp_rn(s);
    codes = make_uint2(0u, 0u);
    if (scale == 0 || nan) return scale;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        codes.x |= encode_two(x[2 * i] * unit_inv, x[2 * i + 1] * unit_inv, s, inv) << (8 * i);
        codes.y |= encode_two(x[8 + 2 * i] * unit_inv, x[9 + 2 * i] * unit_inv, s, inv) << (8 * i);
    }
    return scale;
}

// A thread encodes a group of a token's key row and the same of its value row.
template <typename T, bool VEC>
__global__ void __launch_bounds__(C4_THREADS) cache4_append_kernel(const Append4Args a) {
    const CacheView& v = a.f.v;
    const int chain = blockIdx.z, g = blockIdx.y, c = chain / v.L, l = chain % v.L;
    pdl_wait();
    const int len = cache_len(v, c);
    const int n = a.counts ? min(max(a.counts[c], 0), a.n_tok) : a.n_tok;
    if (a.lens_out && blockIdx.x == 0 && g == 0 && l == 0 && threadIdx.x == 0) a.lens_out[c] = (int)min((long long)len + n, v.cap);
    const long long e = (long long)blockIdx.x * C4_THREADS + threadIdx.x;
    const int i = (int)(e / a.groups), u = (int)(e % a.groups);
    if (i >= n) return;
    const long long pos = (long long)len + i;
    if (pos >= v.cap) {
        cache_fail(v.status, DS_CACHE_LEN);
        return;
    }
    if (u == 0 && v.score) v.score[(((size_t)c * v.Lh + l) * v.n_kv + g) * v.cap + pos] = 0.f;
    const int page = cache_page(v, v.table + (size_t)c * v.width, (int)(pos >> v.page_log2));
    if (page < 0) return;
    const long long src = c * a.s0 + l * a.s1 + g * a.s2 + i * a.s3 + 16 * u;
    float k[16], w[16];
    load16<T, VEC>(static_cast<const T*>(a.K) + src, k);
    load16<T, VEC>(static_cast<const T*>(a.V) + src, w);
    const FourRows rows(a.f, l, g);
    const long long code = rows.code(page, (int)pos) + 8 * u, scale = rows.scale(page, (int)pos) + u;
    uint2 q;
    rows.Ks[scale] = (uint8_t)encode16(k, a.k_inv, q);
    *reinterpret_cast<uint2*>(rows.K + code) = q;
    rows.Vs[scale] = (uint8_t)encode16(w, a.v_inv, q);
    *reinterpret_cast<uint2*>(rows.V + code) = q;
}

template <typename T, bool VEC>
cudaError_t append(const Append4Args& a, cudaStream_t st) {
    const dim3 grid((unsigned)(((long long)a.n_tok * a.groups + C4_THREADS - 1) / C4_THREADS), a.f.v.n_kv, a.f.v.n_ctx * a.f.v.L);
    return launch_kernel(cache4_append_kernel<T, VEC>, grid, dim3(C4_THREADS), 0, st, true, 1, a);
}

// ---------------------------------------------------------------- read
struct Read4Args {
    Cache4View f;
    void *K, *V;
    long long s0, s1, s2, s3;  // element strides (context, layer, head, place)
    int n_pos, units;          // eights of a row
    const int* from;
};

template <typename T, bool VEC>
__device__ __forceinline__ void store8(T* p, const float (&x)[8]) {
    if constexpr (VEC) {
        T t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = from_f<T>(x[i]);
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(p)[i] = reinterpret_cast<const uint4*>(t)[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = from_f<T>(x[i]);
    }
}
__device__ __forceinline__ void decode8(uint32_t codes, float scale, float (&x)[8]) {
    uint32_t h[4];
    code_halves(codes, h);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 two = halves_float2(h[i]);
        x[2 * i] = two.x * scale;
        x[2 * i + 1] = two.y * scale;
    }
}

// A thread decodes eight elements of a position's key row and the same of its value row.
template <typename T, bool VEC>
__global__ void __launch_bounds__(C4_THREADS) cache4_read_kernel(const Read4Args a) {
    const CacheView& v = a.f.v;
    const int chain = blockIdx.z, g = blockIdx.y, c = chain / v.L, l = chain % v.L;
    pdl_wait();
    const long long e = (long long)blockIdx.x * C4_THREADS + threadIdx.x;
    const int i = (int)(e / a.units), u = (int)(e % a.units);
    if (i >= a.n_pos) return;
    const long long pos = (long long)(a.from ? max(a.from[c], 0) : 0) + i;
    if (pos >= cache_len(v, c)) return;
    const int page = cache_page(v, v.table + (size_t)c * v.width, (int)(pos >> v.page_log2));
    if (page < 0) return;
    const FourRows rows(a.f, l, g);
    const long long code = rows.code(page, (int)pos) + 4 * u, scale = rows.scale(page, (int)pos) + (u >> 1);
    const uint32_t kc = *reinterpret_cast<const uint32_t*>(rows.K + code), vc = *reinterpret_cast<const uint32_t*>(rows.V + code);
    const float ks = scale_float(rows.Ks[scale]) * a.f.k_unit, vs = scale_float(rows.Vs[scale]) * a.f.v_unit;
    const long long dst = c * a.s0 + l * a.s1 + g * a.s2 + i * a.s3 + 8 * u;
    float x[8];
    decode8(kc, ks, x);
    store8<T, VEC>(static_cast<T*>(a.K) + dst, x);
    decode8(vc, vs, x);
    store8<T, VEC>(static_cast<T*>(a.V) + dst, x);
}

template <typename T, bool VEC>
cudaError_t read(const Read4Args& a, cudaStream_t st) {
    const dim3 grid((unsigned)(((long long)a.n_pos * a.units + C4_THREADS - 1) / C4_THREADS), a.f.v.n_kv, a.f.v.n_ctx * a.f.v.L);
    return launch_kernel(cache4_read_kernel<T, VEC>, grid, dim3(C4_THREADS), 0, st, true, 1, a);
}

// ---------------------------------------------------------------- eviction: the survivors' rows
struct Evict4Args {
    Cache4View f;
    int keep;
    const int* to;
    int to_width;
    long long to_cap;
    float* to_score;
    const int* kept;
};
constexpr int CM4_SLOTS = 8;

// A warp takes CM4_SLOTS survivors: a lane looks up where one comes from and goes to and moves its scales, then all move 16 bytes of codes each.
template <int HD>
__global__ void __launch_bounds__(C4_THREADS) cache4_compact_kernel(const Evict4Args a) {
    constexpr int UNITS = HD / 32;  // of 16 bytes, of a row's codes
    using Scales = typename std::conditional<HD == 64, uint32_t, uint2>::type;
    const CacheView& v = a.f.v;
    const int chain = blockIdx.z, g = blockIdx.y, c = chain / v.L, l = chain % v.L, lane = threadIdx.x & 31;
    const int i0 = (blockIdx.x * (C4_THREADS / 32) + (threadIdx.x >> 5)) * CM4_SLOTS;
    pdl_wait();
    if (i0 >= a.keep) return;
    const FourRows rows(a.f, l, g);
    long long src = -1, dst = -1;
    const int i = i0 + lane;
    if (lane < CM4_SLOTS && i < a.keep) {
        const int from = a.kept[((size_t)chain * v.n_kv + g) * a.keep + i];
        if (from >= 0) {  // (past the survivors, an entry of the target's table need not name a page)
            const int p1 = cache_page(v, a.to + (size_t)c * a.to_width, i >> v.page_log2);
            const size_t row = ((size_t)c * v.Lh + l) * v.n_kv + g;
            const int p0 = cache_page(v, v.table + (size_t)c * v.width, from >> v.page_log2);
            a.to_score[row * a.to_cap + i] = v.score[row * v.cap + from];
            if (p0 >= 0 && p1 >= 0) {
                src = rows.code(p0, from);
                dst = rows.code(p1, i);
                const long long s = rows.scale(p0, from), d = rows.scale(p1, i);
                const Scales ks = *reinterpret_cast<const Scales*>(rows.Ks + s), vs = *reinterpret_cast<const Scales*>(rows.Vs + s);
                *reinterpret_cast<Scales*>(rows.Ks + d) = ks;
                *reinterpret_cast<Scales*>(rows.Vs + d) = vs;
            }
        }
    }
    // of a slot its key row's units, then its value row's
    for (int e = lane; e < CM4_SLOTS * 2 * UNITS; e += 32) {
        const int slot = e / (2 * UNITS), o = 16 * (e % UNITS);
        const long long s = __shfl_sync(0xffffffffu, src, slot), d = __shfl_sync(0xffffffffu, dst, slot);
        uint8_t* const p = e / UNITS & 1 ? rows.V : rows.K;
        if (s >= 0) *reinterpret_cast<uint4*>(p + d + o) = *reinterpret_cast<const uint4*>(p + s + o);
    }
}

template <int HD>
cudaError_t compact(const Evict4Args& a, cudaStream_t st) {
    const int slots = CM4_SLOTS * C4_THREADS / 32;
    const dim3 grid((unsigned)((a.keep + slots - 1) / slots), a.f.v.n_kv, a.f.v.n_ctx * a.f.v.L);
    return launch_kernel(cache4_compact_kernel<HD>, grid, dim3(C4_THREADS), 0, st, true, 1, a);
}

// Whether rows of T at p with these element strides start on 16-byte boundaries
bool vec_rows(const void* K, const void* V, const long long* strides, int el) {
    uintptr_t all = (uintptr_t)K | (uintptr_t)V;
    for (int i = 0; i < 4; ++i) all |= (uintptr_t)(strides[i] * el);
    return (all & 15u) == 0;
}

}  // namespace

cudaError_t launch_cache4_append(const DevState& s, const Cache4View& f, const void* K, const void* V, const long long* strides, int n_tok,
                                 const int* counts, int* lens_out, cudaStream_t st) {
    const Append4Args a{f, K, V, strides[0], strides[1], strides[2], strides[3], n_tok, s.hd / 16, 1.f / f.k_unit, 1.f / f.v_unit, counts, lens_out};
    const bool vec = vec_rows(K, V, strides, s.dtype == 0 ? 4 : 2);
    if (s.dtype == 0) return vec ? append<float, true>(a, st) : append<float, false>(a, st);
    return vec ? append<bf16, true>(a, st) : append<bf16, false>(a, st);
}

cudaError_t launch_cache4_read(const DevState& s, const Cache4View& f, const int* from, int n_pos, void* K, void* V, const long long* strides,
                               cudaStream_t st) {
    const Read4Args a{f, K, V, strides[0], strides[1], strides[2], strides[3], n_pos, s.hd / 8, from};
    const bool vec = vec_rows(K, V, strides, s.dtype == 0 ? 4 : 2);
    if (s.dtype == 0) return vec ? read<float, true>(a, st) : read<float, false>(a, st);
    return vec ? read<bf16, true>(a, st) : read<bf16, false>(a, st);
}

cudaError_t launch_cache4_evict(const DevState& s, const Cache4View& f, int keep, int n_sink, int n_recent, const int* to, int to_width,
                                float* to_score, int* kept, int* lens_out, cudaStream_t st) {
    const cudaError_t e = launch_cache_select(s, f.v, keep, n_sink, n_recent, kept, lens_out, st);
    if (e != cudaSuccess) return e;
    const Evict4Args a{f, keep, to, to_width, (long long)to_width << f.v.page_log2, to_score, kept};
    return s.hd == 64 ? compact<64>(a, st) : compact<128>(a, st);
}

}  // namespace mone
