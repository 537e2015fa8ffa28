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
    int n_tok;
    float k_inv, v_inv;        // 2^-exp
    const int* counts;
    int* lens_out;
};

// 16 neighbours as they are
template <typename T, bool VEC>
struct Group {
    static constexpr int WORDS = 16 * sizeof(T) / 4;
    uint32_t w[WORDS];
    __device__ __forceinline__ void load(const T* p) {
        if constexpr (VEC) {
#pragma unroll
            for (int i = 0; i < WORDS; i += 8)
                asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                             : "=r"(w[i]), "=r"(w[i + 1]), "=r"(w[i + 2]), "=r"(w[i + 3]), "=r"(w[i + 4]), "=r"(w[i + 5]), "=r"(w[i + 6]), "=r"(w[i + 7])
                             : "l"(reinterpret_cast<const uint32_t*>(p) + i));
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) reinterpret_cast<T*>(w)[i] = p[i];
        }
    }
};

// A group's 16 codes (two words) and its scale.  Of 32-bit values the codes are those of the quotients rounded so that no tie is made or lost.
template <bool VEC>
__device__ __forceinline__ uint32_t encode16(const Group<float, VEC>& x, float unit_inv, uint2& codes) {
    float most = 0.f, v[16];
    bool nan = false;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        v[i] = __uint_as_float(x.w[i]) * unit_inv;
        most = fmaxf(most, fabsf(v[i]));
        nan |= isnan(v[i]);
    }
    const uint32_t scale = nan ? 0x7fu : encode_scale(most);
    codes = make_uint2(0u, 0u);
    if (scale == 0 || nan) return scale;
    const float s = scale_float(scale), inv = __frcp_rn(s);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        codes.x |= encode_two(v[2 * i], v[2 * i + 1], s, inv) << (8 * i);
        codes.y |= encode_two(v[8 + 2 * i], v[9 + 2 * i], s, inv) << (8 * i);
    }
    return scale;
}
// Of bf16 values, 8 bits, and a scale of 4 bits, a quotient that is no tie (of 3 bits) is 2^-9 of itself away from one at least, so its rounding to a
// grid of 2^-13, by a sum with 1.5 x 2^10, gives ties where there are any and moves nothing over one: 3 instructions a value for 9.
template <bool VEC>
__device__ __forceinline__ uint32_t encode16(const Group<bf16, VEC>& x, float unit_inv, uint2& codes) {
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = __vmaxu2(most, x.w[i] & 0x7fff7fffu);
    most = max(most & 0xffffu, most >> 16);
    const bool nan = most > 0x7f80u;
    const uint32_t scale = nan ? 0x7fu : encode_scale(__uint_as_float(most << 16) * unit_inv);
    codes = make_uint2(0u, 0u);
    if (scale == 0 || nan) return scale;
    const float inv = __frcp_rn(scale_float(scale)) * unit_inv;
    uint32_t c[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float2 v = make_float2(__uint_as_float(x.w[i] << 16), __uint_as_float(x.w[i] & 0xffff0000u));
        const float2 q = add2(fma2(v, make_float2(inv, inv), make_float2(1536.f, 1536.f)), make_float2(-1536.f, -1536.f));
        c[i] = code_two(copysignf(q.x, v.x), copysignf(q.y, v.y));
    }
    codes = make_uint2(__byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410),
                       __byte_perm(__byte_perm(c[4], c[5], 0x0040), __byte_perm(c[6], c[7], 0x0040), 0x5410));
    return scale;
}

// A thread encodes PER groups of a token's key row and the same of its value row.  Bound by instructions where there are many tokens, 430 a group of
// both: 2048 tokens of 16 layers, 8 heads of 64, in 20.2 us, 86 MB at 4.3 TB/s (31 with quotients as for 32 bits); two groups of bf16
// values a thread, which share the addresses, 345 and 19.7.  A token a context is bound by the launch and two dependent loads: with its read 3.6 us in a
// graph, by two groups a thread 4.0.
template <typename T, int HD, bool VEC, int PER>
__global__ void __launch_bounds__(C4_THREADS) cache4_append_kernel(const Append4Args a) {
    constexpr int EACH = HD / (16 * PER);  // threads of a row
    using Codes = typename std::conditional<PER == 2, uint4, uint2>::type;
    using Scales = typename std::conditional<PER == 2, uint16_t, uint8_t>::type;
    const CacheView& v = a.f.v;
    const int chain = blockIdx.z, g = blockIdx.y, c = chain / v.L, l = chain % v.L;
    pdl_wait();
    const int len = cache_len(v, c);
    const int n = a.counts ? min(max(a.counts[c], 0), a.n_tok) : a.n_tok;
    if (a.lens_out && blockIdx.x == 0 && g == 0 && l == 0 && threadIdx.x == 0) a.lens_out[c] = (int)min((long long)len + n, v.cap);
    const int i = blockIdx.x * (C4_THREADS / EACH) + threadIdx.x / EACH, u = threadIdx.x % EACH;
    if (i >= n) return;
    const int pos = len + i;  // at most 2^30 + 2^20
    if (pos >= v.cap) {
        cache_fail(v.status, DS_CACHE_LEN);
        return;
    }
    if (u == 0 && v.score) v.score[(((size_t)c * v.Lh + l) * v.n_kv + g) * v.cap + pos] = 0.f;
    const long long src = c * a.s0 + l * a.s1 + g * a.s2 + i * a.s3 + 16 * PER * u;
    Group<T, VEC> k[PER], w[PER];
#pragma unroll
    for (int y = 0; y < PER; ++y) {
        k[y].load(static_cast<const T*>(a.K) + src + 16 * y);
        w[y].load(static_cast<const T*>(a.V) + src + 16 * y);
    }
    const int page = cache_page(v, v.table + (size_t)c * v.width, pos >> v.page_log2);
    if (page < 0) return;
    const FourRows rows(a.f, l, g);
    const long long code = rows.code(page, pos) + 8 * PER * u, scale = rows.scale(page, pos) + PER * u;
    auto put = [&](const Group<T, VEC>(&x)[PER], float unit_inv, uint8_t* codes, uint8_t* scales) {
        __align__(16) uint2 q[PER];
        uint32_t s = 0;
#pragma unroll
        for (int y = 0; y < PER; ++y) s |= encode16(x[y], unit_inv, q[y]) << (8 * y);
        *reinterpret_cast<Scales*>(scales) = (Scales)s;
        *reinterpret_cast<Codes*>(codes) = *reinterpret_cast<const Codes*>(q);
    };
    put(k, a.k_inv, rows.K + code, rows.Ks + scale);
    put(w, a.v_inv, rows.V + code, rows.Vs + scale);
}

template <typename T, int HD, int PER>
cudaError_t append(const Append4Args& a, bool vec, cudaStream_t st) {
    const int tokens = C4_THREADS / (HD / 16) * PER;
    const dim3 grid((unsigned)((a.n_tok + tokens - 1) / tokens), a.f.v.n_kv, a.f.v.n_ctx * a.f.v.L);
    return vec ? launch_kernel(cache4_append_kernel<T, HD, true, PER>, grid, dim3(C4_THREADS), 0, st, true, 1, a)
               : launch_kernel(cache4_append_kernel<T, HD, false, PER>, grid, dim3(C4_THREADS), 0, st, true, 1, a);
}
template <typename T, int HD>
cudaError_t append(const Append4Args& a, bool vec, int sms, cudaStream_t st) {
    if constexpr (sizeof(T) == 2) {  // two groups a thread where that leaves every SM its threads
        const long long threads = (long long)a.n_tok * a.f.v.n_kv * a.f.v.n_ctx * a.f.v.L * (HD / 32);
        if (threads >= 2048ll * sms) return append<T, HD, 2>(a, vec, st);
    }
    return append<T, HD, 1>(a, vec, st);
}

// ---------------------------------------------------------------- read
struct Read4Args {
    Cache4View f;
    void *K, *V;
    long long s0, s1, s2, s3;  // element strides (context, layer, head, place)
    int n_pos;
    const int* from;
};

// 16 values of their codes and scale.  A code's product with its scale is exact in a half, and that times 2^exp in T.
template <typename T, bool VEC>
__device__ __forceinline__ void decode16(T* p, uint2 codes, uint32_t scale, float unit) {
    uint32_t h[8];
    code_halves(codes.x, *reinterpret_cast<uint32_t(*)[4]>(h));
    code_halves(codes.y, *reinterpret_cast<uint32_t(*)[4]>(h + 4));
    const uint32_t s = scale_halves(scale * 0x101u);
    __align__(16) T t[16];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float2 x = mul2(halves_float2(mul_halves(h[i], s)), make_float2(unit, unit));
        if constexpr (sizeof(T) == 2) {
            reinterpret_cast<uint32_t*>(t)[i] = pack_bf16(x.x, x.y);
        } else {
            t[2 * i] = x.x;
            t[2 * i + 1] = x.y;
        }
    }
    if constexpr (VEC) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) st_32b(reinterpret_cast<bf16*>(p) + 16 * i, reinterpret_cast<const uint32_t*>(t) + 8 * i);
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) p[i] = t[i];
    }
}

// A thread decodes a group of a position's key row and the same of its value row: 385 thousand rows of 128 twice in 41 us, 252 MB at 6.1 TB/s.
// (Eight elements a thread in stores of 16 bytes were bound by instructions, 61 us.)
template <typename T, int HD, bool VEC>
__global__ void __launch_bounds__(C4_THREADS) cache4_read_kernel(const Read4Args a) {
    constexpr int GROUPS = HD / 16;
    const CacheView& v = a.f.v;
    const int chain = blockIdx.z, g = blockIdx.y, c = chain / v.L, l = chain % v.L;
    pdl_wait();
    const int i = blockIdx.x * (C4_THREADS / GROUPS) + threadIdx.x / GROUPS, u = threadIdx.x % GROUPS;
    const long long at = (long long)(a.from ? max(a.from[c], 0) : 0) + i;
    if (i >= a.n_pos || at >= cache_len(v, c)) return;
    const int pos = (int)at, page = cache_page(v, v.table + (size_t)c * v.width, pos >> v.page_log2);
    if (page < 0) return;
    const FourRows rows(a.f, l, g);
    const long long code = rows.code(page, pos) + 8 * u, scale = rows.scale(page, pos) + u;
    const uint2 kc = *reinterpret_cast<const uint2*>(rows.K + code), vc = *reinterpret_cast<const uint2*>(rows.V + code);
    const uint32_t ks = rows.Ks[scale], vs = rows.Vs[scale];
    const long long dst = c * a.s0 + l * a.s1 + g * a.s2 + i * a.s3 + 16 * u;
    decode16<T, VEC>(static_cast<T*>(a.K) + dst, kc, ks, a.f.k_unit);
    decode16<T, VEC>(static_cast<T*>(a.V) + dst, vc, vs, a.f.v_unit);
}

template <typename T, int HD>
cudaError_t read(const Read4Args& a, bool vec, cudaStream_t st) {
    const int places = C4_THREADS / (HD / 16);
    const dim3 grid((unsigned)((a.n_pos + places - 1) / places), a.f.v.n_kv, a.f.v.n_ctx * a.f.v.L);
    return vec ? launch_kernel(cache4_read_kernel<T, HD, true>, grid, dim3(C4_THREADS), 0, st, true, 1, a)
               : launch_kernel(cache4_read_kernel<T, HD, false>, grid, dim3(C4_THREADS), 0, st, true, 1, a);
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

// A warp takes 32 survivors: a lane looks up where one comes from and goes to and moves its scales, then all move 16 bytes of codes each, four under
// way at a time.  385 thousand rows of 72 bytes twice, read and written, in 22 us, 5 TB/s (8 survivors a warp: 31).
template <int HD>
__global__ void __launch_bounds__(C4_THREADS) cache4_compact_kernel(const Evict4Args a) {
    constexpr int UNITS = HD / 32, AHEAD = 4;  // 16 bytes of a row's codes; loads under way
    using Scales = typename std::conditional<HD == 64, uint32_t, uint2>::type;
    const CacheView& v = a.f.v;
    const int chain = blockIdx.z, g = blockIdx.y, c = chain / v.L, l = chain % v.L, lane = threadIdx.x & 31;
    const int i0 = blockIdx.x * C4_THREADS + (threadIdx.x & ~31), i = i0 + lane;
    pdl_wait();
    if (i0 >= a.keep) return;
    const FourRows rows(a.f, l, g);
    long long src = -1, dst = -1;
    const int from = i < a.keep ? a.kept[((size_t)chain * v.n_kv + g) * a.keep + i] : -1;
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
    // of a slot its key row's units, then its value row's: a lane the same unit of every slot that it moves
    const int o = 16 * (lane % UNITS), slot0 = lane / (2 * UNITS);
    uint8_t* const p = (lane / UNITS & 1 ? rows.V : rows.K) + o;
#pragma unroll 1
    for (int x = 0; x < 2 * UNITS; x += AHEAD) {
        uint4 moved[AHEAD];
        long long d[AHEAD];
#pragma unroll
        for (int y = 0; y < AHEAD; ++y) {
            const int slot = (x + y) * (16 / UNITS) + slot0;
            const long long s = __shfl_sync(0xffffffffu, src, slot);
            d[y] = __shfl_sync(0xffffffffu, dst, slot);
            if (s < 0)
                d[y] = -1;
            else
                moved[y] = *reinterpret_cast<const uint4*>(p + s);
        }
#pragma unroll
        for (int y = 0; y < AHEAD; ++y)
            if (d[y] >= 0) *reinterpret_cast<uint4*>(p + d[y]) = moved[y];
    }
}

template <int HD>
cudaError_t compact(const Evict4Args& a, cudaStream_t st) {
    const dim3 grid((unsigned)((a.keep + C4_THREADS - 1) / C4_THREADS), a.f.v.n_kv, a.f.v.n_ctx * a.f.v.L);
    return launch_kernel(cache4_compact_kernel<HD>, grid, dim3(C4_THREADS), 0, st, true, 1, a);
}

// Whether rows of T at p with these element strides start on 32-byte boundaries
bool vec_rows(const void* K, const void* V, const long long* strides, int el) {
    uintptr_t all = (uintptr_t)K | (uintptr_t)V;
    for (int i = 0; i < 4; ++i) all |= (uintptr_t)(strides[i] * el);
    return (all & 31u) == 0;
}

}  // namespace

cudaError_t launch_cache4_append(const DevState& s, const Cache4View& f, const void* K, const void* V, const long long* strides, int n_tok,
                                 const int* counts, int* lens_out, cudaStream_t st) {
    const Append4Args a{f, K, V, strides[0], strides[1], strides[2], strides[3], n_tok, 1.f / f.k_unit, 1.f / f.v_unit, counts, lens_out};
    const bool vec = vec_rows(K, V, strides, s.dtype == 0 ? 4 : 2);
    if (s.dtype == 0) return s.hd == 64 ? append<float, 64>(a, vec, s.sms, st) : append<float, 128>(a, vec, s.sms, st);
    return s.hd == 64 ? append<bf16, 64>(a, vec, s.sms, st) : append<bf16, 128>(a, vec, s.sms, st);
}

cudaError_t launch_cache4_read(const DevState& s, const Cache4View& f, const int* from, int n_pos, void* K, void* V, const long long* strides,
                               cudaStream_t st) {
    const Read4Args a{f, K, V, strides[0], strides[1], strides[2], strides[3], n_pos, from};
    const bool vec = vec_rows(K, V, strides, s.dtype == 0 ? 4 : 2);
    if (s.dtype == 0) return s.hd == 64 ? read<float, 64>(a, vec, st) : read<float, 128>(a, vec, st);
    return s.hd == 64 ? read<bf16, 64>(a, vec, st) : read<bf16, 128>(a, vec, st);
}

cudaError_t launch_cache4_evict(const DevState& s, const Cache4View& f, int keep, int n_sink, int n_recent, const int* to, int to_width,
                                float* to_score, int* kept, int* lens_out, cudaStream_t st) {
    const cudaError_t e = launch_cache_select(s, f.v, keep, n_sink, n_recent, kept, lens_out, st);
    if (e != cudaSuccess) return e;
    const Evict4Args a{f, keep, to, to_width, (long long)to_width << f.v.page_log2, to_score, kept};
    return s.hd == 64 ? compact<64>(a, st) : compact<128>(a, st);
}

}  // namespace mone
