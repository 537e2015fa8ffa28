// Attention of each context's newest tokens over its paged cache (mone_cache_attention), and the weights that the cache's
// positions are given by it.
//
// Every context's visible positions are cut into blocks of 32, and the blocks of all (context, layer, KV head, row tile)
// items, one item after the other, are dealt out evenly to a grid that fills the GPU once: however unequal the contexts
// are, every CTA reads as much as any other, and nothing of it has to be known on the host.  A CTA's warps take an item's
// blocks in turn, each with a softmax of its own, and meet in shared memory.  An item that one CTA has whole is
// written at once; the parts of others go to the workspace, and the CTA that finishes an item's last part joins
// them in order, so the result does not depend on who comes last.
//
// For the weights the scores go to the workspace as well, and a second kernel turns them into exp(z - max) / sum,
// summed over the rows of a KV head: 4 bytes a row and position beside the 4 head_dim (bf16) of its key and value.
#include <algorithm>
#include <climits>

#include "cache_common.cuh"
#include "per_device.h"

namespace mone {

namespace {

constexpr int CA_WARPS = 4, CA_THREADS = CA_WARPS * 32;
constexpr int KB = 32;         // positions of a block
constexpr int CA_CTAS = 4;     // CTAs an SM at most
constexpr int CA_WHOLE = 8;    // items of up to so many blocks are not split

struct CaArgs {
    CacheView v;
    const void* Q;             // [chains][n_q][n_tok][hd]: the rows (head of the group, token) of a KV head are contiguous
    void* out;
    int n_tok, R, RT, n_sink, window;  // rows and row tiles of a KV head
    long long per;             // items of a context
    int vec;                   // 16-byte aligned rows
    float scale;
    int* count;                // [grid] parts done of the item that is split from this CTA on; zero between calls
    float* part;               // [2 grid][ROWS][hd + 3]
    float* lse;                // [chains][n_kv][R] log2 of the sum of exp, with the weights
    float* z2;                 // [chains][n_kv][R][pitch] scores in base 2, -inf where not seen
    long long pitch;
};

// 2^x on the special-function unit, error below 2^-22 of the result
__device__ __forceinline__ float ca_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// What the tokens of a context see: blocks of the first positions, then from the oldest token's window on
struct CaRange {
    int n, t0, ns, lo, nb;  // positions held; the oldest token's; blocks of the first; first position after them; blocks
    __device__ CaRange() {}
    __device__ CaRange(const CaArgs& a, int c) {
        n = cache_len(a.v, c);
        t0 = max(0, n - a.n_tok);
        ns = (min(a.n_sink, n) + KB - 1) / KB;
        lo = max(ns * KB, (t0 - a.window + 1) & ~(KB - 1));
        nb = ns + (lo < n ? (n - lo + KB - 1) / KB : 0);
    }
    __device__ int at(int b) const { return b < ns ? b * KB : lo + (b - ns) * KB; }
    __device__ int units() const { return max(nb, 1); }  // an item without a block still writes its zeros
};

// The share of a CTA: units [begin, end), from unit `at0` of context `c` on
struct CaShare {
    long long share, begin, end, ctx0;  // ctx0: first unit of context c
    int c;
    // where unit u lies: the first unit of its context, and the context
    static __device__ void locate(const CaArgs& a, long long u, long long& base, int& c) {
        const int lane = threadIdx.x & 31;
        base = 0;
        for (int c0 = 0;; c0 += 32) {
            const long long mine = c0 + lane < a.v.n_ctx ? CaRange(a, c0 + lane).units() * a.per : 0;
            long long incl = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long up = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += up;
            }
            const uint32_t past = __ballot_sync(0xffffffffu, base + incl > u);
            if (past || c0 + 32 >= a.v.n_ctx) {
                const int k = past ? __ffs(past) - 1 : 31;
                c = c0 + k;
                base += __shfl_sync(0xffffffffu, incl - mine, k);
                return;
            }
            base += __shfl_sync(0xffffffffu, incl, 31);
        }
    }
    // a boundary between CTAs: in an item that stays whole, its start
    static __device__ long long snap(const CaArgs& a, long long u, long long total) {
        if (u >= total) return total;
        long long base;
        int c;
        locate(a, u, base, c);
        const int un = CaRange(a, c).units();
        return un <= CA_WHOLE ? base + (u - base) / un * un : u;
    }
    __device__ CaShare(const CaArgs& a) {
        long long total = 0;
        for (int c0 = threadIdx.x & 31; c0 < a.v.n_ctx; c0 += 32) total += CaRange(a, c0).units() * a.per;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
        share = max((total + gridDim.x - 1) / gridDim.x, (long long)CA_WARPS);
        begin = snap(a, share * blockIdx.x, total);
        end = snap(a, share * (blockIdx.x + 1), total);
        if (begin < end) locate(a, begin, ctx0, c);
    }
};

// A row of Q over the positions it sees and no others, by one thread: dimensions d0, d0 + 1.  A block's products take a
// value row times a probability of 0 for the rows that do not see it, which is NaN where the value is not finite; only
// with several tokens do the rows of an item differ in what they see.  Reached by non-finite inputs only.
template <typename T, int HD>
__device__ __noinline__ void row_again(const CaArgs& a, const T* q, const T* K, const T* V, const int* table, int vis, int d0, float* o) {
    float m = -INFINITY, l = 0.f;
    o[0] = o[1] = 0.f;
    for (int j = a.n_sink > 0 ? 0 : max(0, vis - a.window); j < vis; ++j) {
        if (j >= a.n_sink && j < vis - a.window) j = vis - a.window;
        if (j >= vis) break;
        const int page = cache_page(a.v, table, j >> a.v.page_log2);
        if (page < 0) continue;
        const long long off = page * a.v.s_page + (j & ((1 << a.v.page_log2) - 1)) * a.v.s_pos;
        float z = 0.f;
        for (int d = 0; d < HD; ++d) z = fmaf(to_f<T>(q[d]), to_f<T>(K[off + d]), z);
        z *= a.scale;
        if (z == -INFINITY) continue;
        const float mn = fmaxf(m, z), corr = __expf(m - mn), p = __expf(z - mn);
        m = mn;
        l = fmaf(l, corr, p);
        o[0] = fmaf(o[0], corr, p * to_f<T>(V[off + d0]));
        o[1] = fmaf(o[1], corr, p * to_f<T>(V[off + d0 + 1]));
    }
    const float inv = l > 0.f ? 1.f / l : l;
    o[0] *= inv;
    o[1] *= inv;
}

template <typename T> __device__ __forceinline__ void store2(T* p, float x, float y);
template <> __device__ __forceinline__ void store2<float>(float* p, float x, float y) { *reinterpret_cast<float2*>(p) = make_float2(x, y); }
template <> __device__ __forceinline__ void store2<bf16>(bf16* p, float x, float y) { *reinterpret_cast<uint32_t*>(p) = pack_bf16(x, y); }

// A part of an item: O [ROWS][HD], then per row the max (of raw scores), the sum that goes with O, and the sum of the
// probabilities before their rounding (for the weights).
template <int HD, int ROWS>
struct Part {
    static constexpr int FLOATS = ROWS * (HD + 3);
};

// An item's rows in the workspace or, joined from `n` parts, in `out`: read(k, i) is element i of part k.
template <typename T, int HD, int ROWS, typename Read>
__device__ __forceinline__ void finish_rows(const CaArgs& a, int n, Read&& read, float* to_part, int rows, float k2, int c, size_t kv, int row0,
                                            const CaRange& r, const T* Kp, const T* Vp) {
    constexpr int ST = ROWS * HD;
    for (int e = 2 * threadIdx.x; e < rows * HD; e += 2 * CA_THREADS) {
        const int row = e / HD, d = e - row * HD;
        float mx = -INFINITY, l = 0.f, lx = 0.f, o0 = 0.f, o1 = 0.f;
        for (int k = 0; k < n; ++k) mx = fmaxf(mx, read(k, ST + row));
#pragma unroll 4
        for (int k = 0; k < n; ++k) {
            const float mk = read(k, ST + row);
            const float f = mk == -INFINITY ? 0.f : ca_exp2((mk - mx) * k2);
            l = fmaf(f, read(k, ST + ROWS + row), l);
            lx = fmaf(f, read(k, ST + 2 * ROWS + row), lx);
            o0 = fmaf(f, read(k, e), o0);
            o1 = fmaf(f, read(k, e + 1), o1);
        }
        if (to_part) {
            __stcg(reinterpret_cast<float2*>(to_part + e), make_float2(o0, o1));
            if (d == 0) {
                __stcg(to_part + ST + row, mx);
                __stcg(to_part + ST + ROWS + row, l);
                __stcg(to_part + ST + 2 * ROWS + row, lx);
            }
            continue;
        }
        const float inv = l == 0.f ? 0.f : 1.f / l;  // no key that counts: 0
        o0 *= inv;
        o1 *= inv;
        const size_t at = kv * a.R + row0 + row;
        if (a.n_tok > 1 && (!isfinite(o0) || !isfinite(o1))) {
            float w[2];
            row_again<T, HD>(a, static_cast<const T*>(a.Q) + at * HD, Kp, Vp, a.v.table + (size_t)c * a.v.width,
                             r.n - a.n_tok + (row0 + row) % a.n_tok + 1, d, w);
            o0 = w[0];
            o1 = w[1];
        }
        store2<T>(static_cast<T*>(a.out) + at * HD + d, o0, o1);
        if (d == 0 && a.lse) a.lse[at] = l == 0.f ? INFINITY : fmaf(mx, k2, log2f(lx));
    }
}

// One CTA's share of the work; Form::piece computes blocks [b0, b1) of an item into the warps' parts.
template <typename Form>
__global__ void __launch_bounds__(CA_THREADS, Form::CTAS) cache_attention_kernel(const CaArgs a) {
    using T = typename Form::T;
    constexpr int HD = Form::HD, ROWS = Form::ROWS, PART = Part<HD, ROWS>::FLOATS;
    extern __shared__ float ca_smem[];
    __shared__ int last;
    const CaShare sh(a);
    if (sh.begin >= sh.end) return;
    const float k2 = a.scale * 1.4426950408889634f;
    long long u = sh.begin, ctx0 = sh.ctx0;
    int c = sh.c;
    CaRange r(a, c);
    while (u < sh.end) {
        const int units = r.units();
        if (u - ctx0 >= units * a.per) {
            ctx0 += units * a.per;
            r = CaRange(a, ++c);
            continue;
        }
        const long long in_ctx = (u - ctx0) / units, item0 = ctx0 + in_ctx * units;
        const int b0 = (int)(u - item0), b1 = (int)min((long long)units, b0 + sh.end - u);
        const int rt = (int)(in_ctx % a.RT);
        const int lg = (int)(in_ctx / a.RT), l = lg / a.v.n_kv, g = lg - l * a.v.n_kv;
        const size_t kv = ((size_t)c * a.v.L + l) * a.v.n_kv + g;
        const int row0 = rt * ROWS, rows = min(ROWS, a.R - row0);
        const T* Kp = static_cast<const T*>(a.v.K) + l * a.v.s_layer + g * a.v.s_head;
        const T* Vp = static_cast<const T*>(a.v.V) + l * a.v.s_layer + g * a.v.s_head;
        Form::piece(a, r, c, kv, row0, rows, Kp, Vp, b0, min(b1, r.nb), k2, ca_smem + (threadIdx.x >> 5) * PART);
        __syncthreads();
        auto mine = [&](int k, int i) { return ca_smem[k * PART + i]; };
        if (b0 == 0 && b1 == units) {
            finish_rows<T, HD, ROWS>(a, CA_WARPS, mine, nullptr, rows, k2, c, kv, row0, r, Kp, Vp);
        } else {
            // slot 1 of a CTA: the first part of an item, which the next CTAs go on with; slot 0: the part it begins with
            float* slot = a.part + (2ll * blockIdx.x + (b0 == 0)) * PART;
            finish_rows<T, HD, ROWS>(a, CA_WARPS, mine, slot, rows, k2, c, kv, row0, r, Kp, Vp);
            const long long first = item0 / sh.share, parts = (item0 + units - 1) / sh.share - first + 1;
            __threadfence();
            __syncthreads();
            int* count = a.count + first;
            if (threadIdx.x == 0) {
                last = atomicAdd(count, 1) == (int)parts - 1;
                if (last) *count = 0;  // for the next call
            }
            __syncthreads();
            if (last) {
                __threadfence();
                const float* p0 = a.part + 2ll * first * PART;
                auto theirs = [&](int k, int i) { return __ldcg(p0 + (2ll * k + (k == 0)) * PART + i); };
                finish_rows<T, HD, ROWS>(a, (int)parts, theirs, nullptr, rows, k2, c, kv, row0, r, Kp, Vp);
            }
        }
        __syncthreads();  // the warps' parts have been read
        u += b1 - b0;
    }
}

// ---------------------------------------------------------------- CUDA cores: fp32, and rows that are not aligned
// Eight lanes share a key, each with head_dim / 8 of its dimensions; the four lane groups of a warp take every fourth key and
// keep a softmax of their own, joined at the end of the piece.
template <typename T_, int HD_>
struct CaCores {
    using T = T_;
    static constexpr int HD = HD_, ROWS = 4, CTAS = HD == 64 ? 3 : 2;
    static constexpr int VE = 16 / sizeof(T), D = HD / 8, NP = D / VE;  // elements of 16 bytes; dimensions and 16-byte pieces of a lane
    static constexpr int U = 2;                                         // keys of a lane group at a time

    static __device__ __forceinline__ void load(const T* row, bool vec, bool in, int l8, float (&f)[D]) {
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const T* s = row + p * 8 * VE + l8 * VE;
            if (!in) {
#pragma unroll
                for (int e = 0; e < VE; ++e) f[p * VE + e] = 0.f;
            } else if (vec) {
                const uint4 x = __ldg(reinterpret_cast<const uint4*>(s));
                const T* t = reinterpret_cast<const T*>(&x);
#pragma unroll
                for (int e = 0; e < VE; ++e) f[p * VE + e] = to_f<T>(t[e]);
            } else {
#pragma unroll
                for (int e = 0; e < VE; ++e) f[p * VE + e] = to_f<T>(s[e]);
            }
        }
    }

    static __device__ __forceinline__ void piece(const CaArgs& a, const CaRange& r, int c, size_t kv, int row0, int rows, const T* Kp,
                                                 const T* Vp, int b0, int b1, float k2, float* part) {
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, grp = lane >> 3, l8 = lane & 7;
        const int* table = a.v.table + (size_t)c * a.v.width;
        const int mask = (1 << a.v.page_log2) - 1;
        float q[ROWS][D], o[ROWS][D], m[ROWS], l[ROWS];
        int vis[ROWS];
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const int row = row0 + min(i, rows - 1);
            load(static_cast<const T*>(a.Q) + (kv * a.R + row) * HD, true, i < rows, l8, q[i]);
            vis[i] = i < rows ? r.n - a.n_tok + row % a.n_tok + 1 : 0;
            m[i] = -INFINITY;
            l[i] = 0.f;
#pragma unroll
            for (int d = 0; d < D; ++d) o[i][d] = 0.f;
        }
        for (int b = b0 + warp; b < b1; b += CA_WARPS) {
            const int j0 = r.at(b);
#pragma unroll 1
            for (int it = 0; it < KB / 4; it += U) {
                float k[U][D], v[U][D], z[U][ROWS];
                int key[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    key[u] = j0 + grp + 4 * (it + u);
                    bool in = key[u] < r.n && (key[u] < a.n_sink || key[u] > r.t0 - a.window);
                    long long off = 0;
                    if (in) {
                        const int page = cache_page(a.v, table, key[u] >> a.v.page_log2);
                        in = page >= 0;
                        off = page * a.v.s_page + (key[u] & mask) * a.v.s_pos;
                    }
                    if (!in) key[u] = INT_MAX;
                    load(Kp + off, a.vec, in, l8, k[u]);
                    load(Vp + off, a.vec, in, l8, v[u]);
                }
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int i = 0; i < ROWS; ++i) {
                        float s = 0.f;
#pragma unroll
                        for (int d = 0; d < D; ++d) s = fmaf(q[i][d], k[u][d], s);
#pragma unroll
                        for (int x = 4; x > 0; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
                        const bool sees = key[u] < vis[i] && (key[u] < a.n_sink || key[u] >= vis[i] - a.window);
                        z[u][i] = sees ? s : -INFINITY;
                    }
                if (a.z2) {  // a row's score by lane 0 .. 3 of the key's group
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        float mine = z[u][0];
#pragma unroll
                        for (int i = 1; i < ROWS; ++i) mine = l8 == i ? z[u][i] : mine;
                        const int at = j0 + grp + 4 * (it + u);
                        if (l8 < rows && at < r.n) a.z2[(kv * a.R + row0 + l8) * a.pitch + at] = mine * k2;
                    }
                }
#pragma unroll
                for (int i = 0; i < ROWS; ++i) {
                    float mn = m[i];
#pragma unroll
                    for (int u = 0; u < U; ++u) mn = fmaxf(mn, z[u][i]);
                    const float corr = mn == -INFINITY ? 1.f : ca_exp2((m[i] - mn) * k2), moff = mn == -INFINITY ? 0.f : -mn * k2;
                    m[i] = mn;
                    float p[U];
                    l[i] *= corr;
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        p[u] = ca_exp2(fmaf(z[u][i], k2, moff));
                        l[i] += p[u];
                    }
#pragma unroll
                    for (int d = 0; d < D; ++d) {
                        o[i][d] *= corr;
#pragma unroll
                        for (int u = 0; u < U; ++u) o[i][d] = fmaf(p[u], v[u][d], o[i][d]);
                    }
                }
            }
        }
        // the lane groups' softmaxes into one
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            float mx = fmaxf(m[i], __shfl_xor_sync(0xffffffffu, m[i], 8));
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
            const float f = m[i] == -INFINITY ? 0.f : ca_exp2((m[i] - mx) * k2);
            l[i] *= f;
            l[i] += __shfl_xor_sync(0xffffffffu, l[i], 8);
            l[i] += __shfl_xor_sync(0xffffffffu, l[i], 16);
#pragma unroll
            for (int d = 0; d < D; ++d) {
                float x = o[i][d] * f;
                x += __shfl_xor_sync(0xffffffffu, x, 8);
                x += __shfl_xor_sync(0xffffffffu, x, 16);
                if (grp == i) part[i * HD + d / VE * 8 * VE + l8 * VE + d % VE] = x;
            }
            if (lane == 0) {
                part[ROWS * HD + i] = mx;
                part[ROWS * (HD + 1) + i] = part[ROWS * (HD + 2) + i] = l[i];
            }
        }
    }
};

// ---------------------------------------------------------------- weights
constexpr int SC_THREADS = 256, SC_POS = 4 * SC_THREADS;

// A thread adds the weights of four positions over the KV head's rows.
__global__ void __launch_bounds__(SC_THREADS) cache_weights_kernel(const CaArgs a) {
    const int chain = blockIdx.z, g = blockIdx.y, c = chain / a.v.L, l = chain % a.v.L;
    const int n = cache_len(a.v, c), p0 = blockIdx.x * SC_POS + 4 * threadIdx.x;
    if (p0 >= n) return;
    const long long t0 = max(0, n - a.n_tok);
    if (p0 >= a.n_sink && p0 + 4 <= t0 - a.window + 1) return;  // nobody sees them
    const size_t kv = (size_t)chain * a.v.n_kv + g;
    float w[4] = {0.f, 0.f, 0.f, 0.f};
    const float* z = a.z2 + kv * a.R * a.pitch + p0;
    const float* lse = a.lse + kv * a.R;
#pragma unroll 4
    for (int row = 0; row < a.R; ++row) {
        const float4 x = __ldcs(reinterpret_cast<const float4*>(z + row * a.pitch));
        const float s = __ldg(lse + row);
        w[0] += ca_exp2(x.x - s);
        w[1] += ca_exp2(x.y - s);
        w[2] += ca_exp2(x.z - s);
        w[3] += ca_exp2(x.w - s);
    }
    float* score = a.v.score + (((size_t)c * a.v.Lh + l) * a.v.n_kv + g) * a.v.cap;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int p = p0 + i;
        if (p < n && (p < a.n_sink || p > t0 - a.window)) score[p] += w[i];
    }
}

template <typename Form>
cudaError_t launch(CaArgs a, int sms, cudaStream_t st) {
    static_assert(Form::CTAS <= CA_CTAS, "the workspace holds the parts of CA_CTAS CTAs an SM");
    if (Form::CTAS * sms > kCacheCounters) return cudaErrorInvalidConfiguration;
    constexpr size_t smem = CA_WARPS * Part<Form::HD, Form::ROWS>::FLOATS * sizeof(float);
    static PerDevice<SmemOptIn> once;
    cudaError_t e = smem_opt_in(reinterpret_cast<const void*>(cache_attention_kernel<Form>), smem, once);
    if (e != cudaSuccess) return e;
    a.RT = (a.R + Form::ROWS - 1) / Form::ROWS;
    a.per = (long long)a.v.L * a.v.n_kv * a.RT;
    cache_attention_kernel<Form><<<Form::CTAS * sms, CA_THREADS, smem, st>>>(a);
    if ((e = cudaGetLastError()) != cudaSuccess || !a.v.score) return e;
    const dim3 grid((unsigned)((a.v.cap + SC_POS - 1) / SC_POS), a.v.n_kv, a.v.n_ctx * a.v.L);
    cache_weights_kernel<<<grid, SC_THREADS, 0, st>>>(a);
    return cudaGetLastError();
}

// The workspace: the counters in the same place whatever the call's sizes, then what a call needs beside them.
struct Layout {
    size_t part, lse, z2, bytes;
    long long pitch;
    Layout(const DevState& s, const CacheView& v, int n_q, int n_tok) {
        const size_t kv = (size_t)v.n_ctx * v.L * v.n_kv, R = (size_t)n_q / v.n_kv * n_tok;
        auto up = [](size_t n) { return (n + 255) / 256 * 256; };
        part = kCacheCounters * sizeof(int);
        lse = part + up((size_t)2 * CA_CTAS * s.sms * Part<128, 16>::FLOATS * sizeof(float));
        z2 = lse + (v.score ? up(kv * R * sizeof(float)) : 0);
        pitch = (v.cap + KB - 1) / KB * KB;
        bytes = z2 + (v.score ? up(kv * R * pitch * sizeof(float)) : 0);
    }
};

}  // namespace

size_t cache_attention_workspace(const DevState& s, const CacheView& v, int n_q, int n_tok) { return Layout(s, v, n_q, n_tok).bytes; }

cudaError_t launch_cache_attention(const DevState& s, const CacheView& v, const void* Q, int n_q, int n_tok, int n_sink, int window,
                                   void* out, void* ws, cudaStream_t st) {
    const Layout w(s, v, n_q, n_tok);
    CaArgs a{};
    a.v = v;
    a.Q = Q; a.out = out;
    a.n_tok = n_tok; a.R = n_q / v.n_kv * n_tok;
    a.n_sink = n_sink; a.window = window;
    a.vec = cache_vec(v, s.dtype == 0 ? 4 : 2);
    a.scale = 1.0f / sqrtf((float)s.hd);
    char* b = static_cast<char*>(ws);
    a.count = reinterpret_cast<int*>(b);
    a.part = reinterpret_cast<float*>(b + w.part);
    a.lse = v.score ? reinterpret_cast<float*>(b + w.lse) : nullptr;
    a.z2 = v.score ? reinterpret_cast<float*>(b + w.z2) : nullptr;
    a.pitch = w.pitch;
    if (s.dtype == 0) return s.hd == 64 ? launch<CaCores<float, 64>>(a, s.sms, st) : launch<CaCores<float, 128>>(a, s.sms, st);
    return s.hd == 64 ? launch<CaCores<bf16, 64>>(a, s.sms, st) : launch<CaCores<bf16, 128>>(a, s.sms, st);
}

}  // namespace mone
