// Attention of each context's newest tokens over its paged cache (mone_cache_attention), and the weights that the cache's
// positions are given by it.
//
// Every context's visible positions are cut into blocks of 32, and the blocks of all (context, layer, KV head, row tile)
// items, one item after the other, are dealt out evenly to the CTAs of a grid that fills the GPU once, and those of a CTA
// to its warps: however unequal the contexts are, every warp reads as much as any other, and nothing of it has to be known on
// the host.  A warp works alone to the end of its share: it keeps an item's softmax and output in registers, and writes the
// rows of an item that it has whole.  Of the others it leaves parts (max, sums and unnormalised output), which the CTA joins
// when its warps are done, to the item's rows if it has the item whole, else to a part that the second kernel
// joins.  Parts are joined in order, so equal calls give equal bits.
//
// Where the items are few and short enough (item_ctas), a cluster takes each of them instead: its CTAs and their warps have equal
// shares of the item's blocks, and at the end they join their parts through distributed shared memory, without a second
// kernel.
//
// For the weights the scores go to the workspace as well (4 bytes a row and position beside the 4 head_dim, in bf16, of its
// key and value), and the second kernel, or the cluster's end, adds exp(z - max) / sum over the rows of a KV head.
#include <algorithm>
#include <climits>
#include <type_traits>

#include "cache_common.cuh"
#include "per_device.h"

namespace mone {

namespace {

constexpr int CA_WARPS = 4, CA_THREADS = CA_WARPS * 32;
constexpr int KB = 32;         // positions of a block
constexpr int CA_WHOLE = 16;   // items of up to so many blocks are not split over CTAs
constexpr int CA_SHARE = 4;    // blocks of a CTA, at least
constexpr int CA_SM_ROWS = 32; // rows of an SM's CTAs, at most
constexpr int FIN_ROWS = 64;   // rows whose weights are added at a time

struct CaArgs {
    CacheView v;
    const void* Q;             // [chains][n_q][n_tok][hd]: the rows (head of the group, token) of a KV head are contiguous
    void* out;
    int n_tok, R, RT, n_sink, window;  // rows and row tiles of a KV head
    int per;                   // items of a context
    int vec;                   // 16-byte aligned rows
    float scale;
    int ctas;                  // that the blocks are dealt out to
    int split;                 // CTAs of an item, or 0: dealt out
    float* part;               // [ctas + 4 ctas][2][ROWS][hd + 3]: the CTAs' parts, and those that their warps put here
    int* info;                 // [chains][n_kv][RT] of an item, the CTA that has its first part and their number (<< 16)
    float* lse;                // [chains][n_kv][R] log2 of the sum of exp of items that one CTA has whole, with the weights
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

__device__ __forceinline__ int udiv(int a, int b) { return (int)((unsigned)a / (unsigned)b); }

// How the units of all items, one item after the other, are dealt out: `share` to each CTA.  A boundary within an item of
// up to CA_WHOLE units moves to the item's start.
struct CaDeal {
    int total, share;
    int units, mine, incl;  // of context c0 + lane, of those scanned last: units of an item, of its items, up to its last
    __device__ CaDeal(const CaArgs& a) {
        total = 0;
        for (int c0 = 0; c0 < a.v.n_ctx; c0 += 32) total = scan(a, c0, total);
        share = max(udiv(total + a.ctas - 1, a.ctas), CA_SHARE);
    }
    // with `before` units ahead of them; returns the units up to the last
    __device__ int scan(const CaArgs& a, int c0, int before) {
        const int lane = threadIdx.x & 31;
        units = c0 + lane < a.v.n_ctx ? CaRange(a, c0 + lane).units() : 0;
        mine = units * a.per;
        incl = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int up = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += up;
        }
        incl += before;
        return __shfl_sync(0xffffffffu, incl, 31);
    }
    // where unit u < total lies: its context, the context's first unit and the units of its items
    __device__ int locate(const CaArgs& a, int u, int& base, int& c) {
        int c0 = 0;
        if (a.v.n_ctx > 32)
            for (int before = scan(a, 0, 0); before <= u; before = scan(a, c0, before)) c0 += 32;
        const int k = __ffs(__ballot_sync(0xffffffffu, incl > u)) - 1;
        c = c0 + k;
        base = __shfl_sync(0xffffffffu, incl - mine, k);
        return __shfl_sync(0xffffffffu, units, k);
    }
    // the first unit of CTA w
    __device__ int start(const CaArgs& a, int w) {
        const int u = w * share;  // below 2^30 + ctas share
        if (u >= total) return total;
        int base, c;
        const int n = locate(a, u, base, c);
        return n <= CA_WHOLE ? base + udiv(u - base, n) * n : u;
    }
};

// The pieces of a warp, one after the other: blocks [b0, b1) of an item
struct CaWalk {
    int u, end, ctx0, c, units;
    CaRange r;
    int l, g, rt, b0, b1;
    int share, parts;         // of a CTA; CTAs that have a part of the item
    bool whole, cta_whole;    // the warp has the item whole, the CTA has
    bool first, last;         // the item begins in the CTA's share; the warp's last piece
    int cta0, cta1;           // the CTA's units
    __device__ CaWalk(const CaArgs& a) {
        const int warp = threadIdx.x >> 5;
        auto share_out = [&]() {
            const int n = cta1 - cta0;
            u = cta0 + n / CA_WARPS * warp + n % CA_WARPS * warp / CA_WARPS;
            end = cta0 + n / CA_WARPS * (warp + 1) + n % CA_WARPS * (warp + 1) / CA_WARPS;
        };
        if (a.split) {  // units as if the item's context were the only one
            const int item = udiv(blockIdx.x, a.split), rank = blockIdx.x - item * a.split;
            c = a.v.n_ctx == 1 ? 0 : udiv(item, a.per);
            r = CaRange(a, c);
            units = r.units();
            ctx0 = 0;
            share = 1;
            const int u0 = (item - c * a.per) * units;
            cta0 = u0 + units * rank / a.split;
            cta1 = u0 + units * (rank + 1) / a.split;
            share_out();
            return;
        }
        CaDeal deal(a);
        share = deal.share;
        cta0 = deal.start(a, blockIdx.x);
        cta1 = deal.start(a, blockIdx.x + 1);
        share_out();
        if (u < end) {
            units = deal.locate(a, u, ctx0, c);
            r = CaRange(a, c);
        }
    }
    __device__ bool next(const CaArgs& a) {
        if (u >= end) return false;
        while (u - ctx0 >= units * a.per) {
            ctx0 += units * a.per;
            r = CaRange(a, ++c);
            units = r.units();
        }
        const int in_ctx = udiv(u - ctx0, units), lg = a.RT == 1 ? in_ctx : udiv(in_ctx, a.RT);
        b0 = u - ctx0 - in_ctx * units;
        const int e = min(units, b0 + end - u);
        whole = b0 == 0 && e == units;
        const int u0 = u - b0;
        cta_whole = u0 >= cta0 && u0 + units <= cta1;
        first = u0 >= cta0;
        parts = cta_whole || !first ? 1 : udiv(u0 + units - 1, share) - udiv(u0, share) + 1;
        b1 = min(e, r.nb);
        u += e - b0;
        last = u >= end;
        rt = in_ctx - lg * a.RT;
        l = a.v.L == 1 ? 0 : udiv(lg, a.v.n_kv);
        g = lg - l * a.v.n_kv;
        return true;
    }
    // index of its KV head's rows, in units of R
    __device__ size_t kv(const CaArgs& a) const { return ((size_t)c * a.v.L + l) * a.v.n_kv + g; }
};

// A row of Q over the positions it sees and no others, by one thread: N dimensions from d0.  A block's products take a
// value row times a probability of 0 for the rows that do not see it, which is NaN where the value is not finite; only
// with several tokens do the rows of an item differ in what they see.  Reached by non-finite inputs only.
template <typename T, int HD, int N>
__device__ __noinline__ void row_again(const CaArgs& a, const T* q, const T* K, const T* V, const int* table, int vis, int d0, float* o) {
    float m = -INFINITY, l = 0.f;
    for (int d = 0; d < N; ++d) o[d] = 0.f;
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
        for (int d = 0; d < N; ++d) o[d] = fmaf(o[d], corr, p * to_f<T>(V[off + d0 + d]));
    }
    const float inv = l > 0.f ? 1.f / l : l;
    for (int d = 0; d < N; ++d) o[d] *= inv;
}

template <typename T> __device__ __forceinline__ void store2(T* p, float x, float y);
template <> __device__ __forceinline__ void store2<float>(float* p, float x, float y) { *reinterpret_cast<float2*>(p) = make_float2(x, y); }
template <> __device__ __forceinline__ void store2<bf16>(bf16* p, float x, float y) { *reinterpret_cast<uint32_t*>(p) = pack_bf16(x, y); }

// A part of an item: O [ROWS][HD], then per row the max (of raw scores), the sum that goes with O, and the sum of the
// probabilities before their rounding (for the weights).  A CTA has two that are not whole, one of the item that it begins
// with in the middle, one of the item that it ends with before its end; a warp the same.
template <int HD, int ROWS>
struct Part {
    static constexpr int FLOATS = ROWS * (HD + 3), M = ROWS * HD, L = M + ROWS, LX = L + ROWS;
    static __device__ float* of_cta(const CaArgs& a, int cta, bool first) { return a.part + (2ll * cta + first) * FLOATS; }
    // of a warp of this CTA
    static __device__ float* of_warp(const CaArgs& a, bool first) {
        return a.part + (2ll * (a.ctas + blockIdx.x * CA_WARPS + (threadIdx.x >> 5)) + first) * FLOATS;
    }
};

// What a warp says of its parts, in the order of their blocks: the piece it begins with, the piece it ends with
struct CaNote {
    const float* part;  // null: no such part
    int c, l, g, rt, n, first, whole;  // the item; positions held; whether the CTA has its first part, all of them
    int parts;                         // of the item, one a CTA
};

// N dimensions from d of a row, from its O and sum, ready to be stored.  (The pools' pointers are their layer's and head's.)
template <typename T, int HD, int N>
__device__ __forceinline__ void finish_row(const CaArgs& a, size_t kv, int c, int n, int row, int d, const T* K, const T* V, float (&o)[N], float l) {
    const float inv = l == 0.f ? 0.f : 1.f / l;  // no key that counts: 0
    bool bad = false;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        o[i] *= inv;
        bad |= !isfinite(o[i]);
    }
    if (a.n_tok > 1 && bad) {
        float w[N];
        row_again<T, HD, N>(a, static_cast<const T*>(a.Q) + (kv * a.R + row) * HD, K, V, a.v.table + (size_t)c * a.v.width,
                            n - a.n_tok + row % a.n_tok + 1, d, w);
#pragma unroll
        for (int i = 0; i < N; ++i) o[i] = w[i];
    }
}
template <typename T, int HD>
__device__ __forceinline__ void write_row(const CaArgs& a, size_t kv, int c, int n, int row, int d, const T* K, const T* V, float o0,
                                          float o1, float l) {
    float o[2] = {o0, o1};
    finish_row<T, HD, 2>(a, kv, c, n, row, d, K, V, o, l);
    store2<T>(static_cast<T*>(a.out) + (kv * a.R + row) * HD + d, o[0], o[1]);
}

// log2 of the sum of exp of a row, +inf where nothing counts (its weights are then 0)
__device__ __forceinline__ float row_lse(float m, float lx, float k2) { return lx == 0.f ? INFINITY : fmaf(m, k2, log2f(lx)); }

// A position's weight from a row.  NANS: some row's sum is not a number; such a row adds nothing where it does not see.  (The
// comparison everywhere: 13.4 us for 12.9 at 16 layers of 1151 positions.)
template <bool NANS>
__device__ __forceinline__ float ca_weight(float z2, float lse) { return NANS && z2 == -INFINITY ? 0.f : ca_exp2(z2 - lse); }

// What the warps of a CTA have of a row's dimensions d and d + 1 (e: their place in a part), in the warps' order
struct CaJoined {
    float mx, l, lx, o0, o1;
    template <typename P>
    static __device__ __forceinline__ CaJoined of(const float* const (&ps)[CA_WARPS], int e, int row, float k2) {
        CaJoined x{-INFINITY, 0.f, 0.f, 0.f, 0.f};
        float mk[CA_WARPS];
#pragma unroll
        for (int k = 0; k < CA_WARPS; ++k) {
            mk[k] = ps[k] ? ps[k][P::M + row] : -INFINITY;
            x.mx = fmaxf(x.mx, mk[k]);
        }
#pragma unroll
        for (int k = 0; k < CA_WARPS; ++k) {
            if (!ps[k]) continue;
            const float f = mk[k] == -INFINITY ? 0.f : ca_exp2((mk[k] - x.mx) * k2);
            const float2 o = *reinterpret_cast<const float2*>(ps[k] + e);
            x.l = fmaf(f, ps[k][P::L + row], x.l);
            x.lx = fmaf(f, ps[k][P::LX + row], x.lx);
            x.o0 = fmaf(f, o.x, x.o0);
            x.o1 = fmaf(f, o.y, x.o1);
        }
        return x;
    }
};

// float (floats) of CTA `rank` of the cluster at the place of `p` in this one
__device__ __forceinline__ float ca_remote(const float* p, uint32_t rank) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(map_to_cta(smem_u32(p), rank)) : "memory");
    return v;
}
__device__ __forceinline__ float2 ca_remote2(const float* p, uint32_t rank) {
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(map_to_cta(smem_u32(p), rank)) : "memory");
    return v;
}

// An item's end where a cluster has it: the CTAs' parts, `mine` in each one's shared memory, are joined through it, each CTA some
// of the dimensions, and each adds its positions' weights.
template <typename Form>
__device__ __forceinline__ void cluster_end(const CaArgs& a, const CaNote* notes, float* mine) {
    using T = typename Form::T;
    constexpr int HD = Form::HD, ROWS = Form::ROWS;
    using P = Part<HD, ROWS>;
    __shared__ float lse[ROWS];
    const float k2 = a.scale * 1.4426950408889634f;
    const int S = a.split, item = udiv(blockIdx.x, S), rank = blockIdx.x - item * S, tid = threadIdx.x;
    const int c = a.v.n_ctx == 1 ? 0 : udiv(item, a.per), in_ctx = item - c * a.per, lg = a.RT == 1 ? in_ctx : udiv(in_ctx, a.RT);
    const int l = a.v.L == 1 ? 0 : udiv(lg, a.v.n_kv), g = lg - l * a.v.n_kv, row0 = (in_ctx - lg * a.RT) * ROWS, rows = min(ROWS, a.R - row0);
    const size_t kv = ((size_t)c * a.v.L + l) * a.v.n_kv + g;
    const CaRange r(a, c);
    const int units = r.units();
    const bool split = S > 1 && units > 1;
    bool nans = false;  // some row's sum
    if (units > 1) {    // else one warp has written the item
        const long long head = l * a.v.s_layer + g * a.v.s_head;
        auto write = [&](int row, int d, float o0, float o1, float l) {
            write_row<T, HD>(a, kv, c, r.n, row0 + row, d, static_cast<const T*>(a.v.K) + head, static_cast<const T*>(a.v.V) + head, o0, o1, l);
        };
        const float* ps[CA_WARPS];
#pragma unroll
        for (int k = 0; k < CA_WARPS; ++k) ps[k] = notes[2 * k].part ? notes[2 * k].part : notes[2 * k + 1].part;
        for (int e = 2 * tid; e < rows * HD; e += 2 * CA_THREADS) {
            const int row = e / HD, d = e - row * HD;
            const auto x = CaJoined::of<P>(ps, e, row, k2);
            if (split) {
                *reinterpret_cast<float2*>(mine + e) = make_float2(x.o0, x.o1);
                if (d == 0) mine[P::M + row] = x.mx, mine[P::L + row] = x.l, mine[P::LX + row] = x.lx;
            } else {
                write(row, d, x.o0, x.o1, x.l);
                if (d == 0) {
                    lse[row] = row_lse(x.mx, x.lx, k2);
                    nans |= isnan(x.lx);
                }
            }
        }
        if (split) {
            cluster_sync();
            // its max over the CTAs, and their factors
            auto factors = [&](int row, float (&f)[8]) {
                float mx = -INFINITY;
#pragma unroll
                for (int k = 0; k < 8; ++k) f[k] = k < S ? ca_remote(mine + P::M + row, k) : -INFINITY;
#pragma unroll
                for (int k = 0; k < 8; ++k) mx = fmaxf(mx, f[k]);
#pragma unroll
                for (int k = 0; k < 8; ++k) f[k] = f[k] == -INFINITY ? 0.f : ca_exp2((f[k] - mx) * k2);
                return mx;
            };
            for (int e = 2 * (tid + rank * CA_THREADS); e < rows * HD; e += 2 * CA_THREADS * S) {
                const int row = e / HD, d = e - row * HD;
                float f[8], lk[8], sum = 0.f, o0 = 0.f, o1 = 0.f;
                float2 o[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    o[k] = k < S ? ca_remote2(mine + e, k) : make_float2(0.f, 0.f);
                    lk[k] = k < S ? ca_remote(mine + P::L + row, k) : 0.f;
                }
                factors(row, f);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    sum = fmaf(f[k], lk[k], sum);
                    o0 = fmaf(f[k], o[k].x, o0);
                    o1 = fmaf(f[k], o[k].y, o1);
                }
                write(row, d, o0, o1, sum);
            }
            if (a.z2 && tid < rows) {
                float f[8], lx = 0.f;
                const float mx = factors(tid, f);
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (k < S) lx = fmaf(f[k], ca_remote(mine + P::LX + tid, k), lx);
                lse[tid] = row_lse(mx, lx, k2);
                nans = isnan(lx);
            }
            asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        }
    } else if (a.z2 && tid < rows) {
        lse[tid] = a.lse[kv * a.R + row0 + tid];
        nans = isnan(lse[tid]);
    }
    if (a.z2) {
        nans = __syncthreads_or(nans);
        const int b0 = units * rank / S, b1 = min(units * (rank + 1) / S, r.nb);
        float* score = a.v.score + (((size_t)c * a.v.Lh + l) * a.v.n_kv + g) * a.v.cap;
        const float* z = a.z2 + (kv * a.R + row0) * a.pitch;
        for (int i = tid; i < (b1 - b0) * (KB / 4); i += CA_THREADS) {  // four positions a thread
            const int p = r.at(b0 + i / (KB / 4)) + i % (KB / 4) * 4;
            bool seen[4];
            float w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                seen[k] = p + k < r.n && (p + k < a.n_sink || p + k > r.t0 - a.window);
                w[k] = seen[k] ? score[p + k] : 0.f;
            }
            float add[4] = {0.f, 0.f, 0.f, 0.f};
            auto sum = [&](auto check) {
                constexpr bool N = decltype(check)::value;
#pragma unroll 4
                for (int row = 0; row < rows; ++row) {
                    const float4 x = *reinterpret_cast<const float4*>(z + row * a.pitch + p);
                    add[0] += ca_weight<N>(x.x, lse[row]);
                    add[1] += ca_weight<N>(x.y, lse[row]);
                    add[2] += ca_weight<N>(x.z, lse[row]);
                    add[3] += ca_weight<N>(x.w, lse[row]);
                }
            };
            nans ? sum(std::true_type()) : sum(std::false_type());
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (seen[k]) score[p + k] = w[k] + add[k];
        }
    }
    if (split) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");  // nobody leaves while another reads its part
}

template <typename Form, bool ITEMS>
__global__ void __launch_bounds__(CA_THREADS, Form::CTAS)
cache_attention_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const CaArgs a) {
    using T = typename Form::T;
    constexpr int HD = Form::HD, ROWS = Form::ROWS;
    using P = Part<HD, ROWS>;
    extern __shared__ uint8_t ca_raw[];
    __shared__ CaNote notes[2 * CA_WARPS];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(ca_raw) + 1023) & ~uintptr_t(1023));
    const int warp = threadIdx.x >> 5;
    if ((threadIdx.x & 31) < 2) notes[2 * warp + (threadIdx.x & 31)].part = nullptr;
    __syncwarp();
    {
        Form form(tmK, tmV, smem + warp * Form::WARP_BYTES, a.RT);
        pdl_wait();
        form.run(a, notes + 2 * warp);
    }
    __syncthreads();
    if constexpr (ITEMS) {
        cluster_end<Form>(a, notes, reinterpret_cast<float*>(smem + CA_WARPS * Form::WARP_BYTES));
        return;
    }
    // the warps' parts, item by item
    const float k2 = a.scale * 1.4426950408889634f;
    for (int i = 0; i < 2 * CA_WARPS;) {
        const CaNote it = notes[i];
        if (!it.part) {
            ++i;
            continue;
        }
        const float* ps[CA_WARPS] = {};
        for (int n = 0; i < 2 * CA_WARPS; ++i) {  // an item's, a warp at most one each
            const CaNote& x = notes[i];
            if (!x.part) continue;
            if (x.c != it.c || x.l != it.l || x.g != it.g || x.rt != it.rt) break;
#pragma unroll
            for (int k = 0; k < CA_WARPS; ++k) ps[k] = k == n ? x.part : ps[k];
            ++n;
        }
        const int row0 = it.rt * ROWS, rows = min(ROWS, a.R - row0);
        const size_t kv = ((size_t)it.c * a.v.L + it.l) * a.v.n_kv + it.g;
        const long long head = it.l * a.v.s_layer + it.g * a.v.s_head;
        if (threadIdx.x == 0 && it.first) a.info[kv * a.RT + it.rt] = blockIdx.x | it.parts << 16;
        float* to = it.whole ? nullptr : P::of_cta(a, blockIdx.x, it.first);
        for (int e = 2 * threadIdx.x; e < rows * HD; e += 2 * CA_THREADS) {
            const int row = e / HD, d = e - row * HD;
            const auto x = CaJoined::of<P>(ps, e, row, k2);
            if (to) {
                *reinterpret_cast<float2*>(to + e) = make_float2(x.o0, x.o1);
                if (d == 0) to[P::M + row] = x.mx, to[P::L + row] = x.l, to[P::LX + row] = x.lx;
            } else {
                write_row<T, HD>(a, kv, it.c, it.n, row0 + row, d, static_cast<const T*>(a.v.K) + head, static_cast<const T*>(a.v.V) + head, x.o0, x.o1,
                                 x.l);
                if (d == 0 && a.lse) a.lse[kv * a.R + row0 + row] = row_lse(x.mx, x.lx, k2);
            }
        }
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
    static constexpr int ONE = 1, EACH = 1, FULL = 1, FEW = 1;          // blocks of a warp, see item_ctas
    static constexpr int WARP_BYTES = 2 * Part<HD, ROWS>::FLOATS * 4;

    float* parts;

    __device__ CaCores(const CUtensorMap&, const CUtensorMap&, uint8_t* smem, int) : parts(reinterpret_cast<float*>(smem)) {}

    __device__ __forceinline__ void run(const CaArgs& a, CaNote* notes) {
        CaWalk walk(a);
        while (walk.next(a)) piece(a, walk, notes);
    }

    static __device__ __forceinline__ void load(const T* row, bool vec, bool in, int l8, float (&f)[D]) {
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const T* s = row + p * 8 * VE + l8 * VE;
            if (!in) {
#pragma unroll
                for (int e = 0; e < VE; ++e) f[p * VE + e] = 0.f;
            } else if (vec) {
                const uint4 x = *reinterpret_cast<const uint4*>(s);
                const T* t = reinterpret_cast<const T*>(&x);
#pragma unroll
                for (int e = 0; e < VE; ++e) f[p * VE + e] = to_f<T>(t[e]);
            } else {
#pragma unroll
                for (int e = 0; e < VE; ++e) f[p * VE + e] = to_f<T>(s[e]);
            }
        }
    }

    __device__ __forceinline__ void piece(const CaArgs& a, const CaWalk& walk, CaNote* notes) {
        const CaRange& r = walk.r;
        const int c = walk.c, row0 = walk.rt * ROWS, rows = min(ROWS, a.R - row0);
        const size_t kv = walk.kv(a);
        const long long head = walk.l * a.v.s_layer + walk.g * a.v.s_head;
        const T *Kp = static_cast<const T*>(a.v.K) + head, *Vp = static_cast<const T*>(a.v.V) + head;
        const float k2 = a.scale * 1.4426950408889634f;
        const int lane = threadIdx.x & 31, grp = lane >> 3, l8 = lane & 7;
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
        for (int b = walk.b0; b < walk.b1; ++b) {
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
        // the lane groups' softmaxes into one; lane group i writes row i
        using P = Part<HD, ROWS>;
        float* part = parts + (walk.b0 == 0) * P::FLOATS;
        if (walk.whole && lane == 0) a.info[kv * a.RT + walk.rt] = 1 << 16;
        if (!walk.whole && lane == 0) notes[walk.b0 == 0] = {part, c, walk.l, walk.g, walk.rt, r.n, walk.first, walk.cta_whole, walk.parts};
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            float mx = fmaxf(m[i], __shfl_xor_sync(0xffffffffu, m[i], 8));
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
            const float f = m[i] == -INFINITY ? 0.f : ca_exp2((m[i] - mx) * k2);
            l[i] *= f;
            l[i] += __shfl_xor_sync(0xffffffffu, l[i], 8);
            l[i] += __shfl_xor_sync(0xffffffffu, l[i], 16);
            if (i >= rows) break;
#pragma unroll
            for (int d = 0; d < D; d += 2) {
                float x[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    x[e] = o[i][d + e] * f;
                    x[e] += __shfl_xor_sync(0xffffffffu, x[e], 8);
                    x[e] += __shfl_xor_sync(0xffffffffu, x[e], 16);
                }
                const int dim = d / VE * 8 * VE + l8 * VE + d % VE;
                if (grp != i) continue;
                if (walk.whole)
                    write_row<T, HD>(a, kv, c, r.n, row0 + i, dim, Kp, Vp, x[0], x[1], l[i]);
                else
                    *reinterpret_cast<float2*>(part + i * HD + dim) = make_float2(x[0], x[1]);
            }
            if (lane == 0) {
                if (!walk.whole)
                    part[P::M + i] = mx, part[P::L + i] = part[P::LX + i] = l[i];
                else if (a.lse)
                    a.lse[kv * a.R + row0 + i] = row_lse(mx, l[i], k2);
            }
        }
    }
};

// ---------------------------------------------------------------- tensor cores: bf16
// A block's keys and values come by TMA, whose box is the positions of a page in the block (a swizzled row of 64 dimensions
// each), into a ring that belongs to one warp: a lane looks up a page and starts its copies, the warp waits for the
// stage, and what it has read is free for the next copy without another warp's say.  The keys are the M of m16n8k16 and
// the rows its N, 8 or 16 of them: S^T = K Q^T by ldmatrix from the key rows, P^T turned in registers (movmatrix), and
// O^T += V^T P^T by transposed ldmatrix.  (The rows as M would have 12 of 16 unused where four heads share a KV head, and a
// 128-row tcgen05 tile 124; what bounds this kernel is the bytes, and at short contexts the chain of a block's steps.)
__device__ __forceinline__ void ca_mma(float (&d)[4], const uint32_t (&A)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(A[0]), "r"(A[1]), "r"(A[2]), "r"(A[3]), "r"(b0), "r"(b1));
}
template <bool TRANS>
__device__ __forceinline__ void ca_ldmatrix(uint32_t (&r)[4], uint32_t addr) {
    if constexpr (TRANS)
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                     : "r"(addr)
                     : "memory");
    else
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                     : "r"(addr)
                     : "memory");
}
// an 8 x 8 matrix of 16-bit elements, two of a row a lane, transposed
__device__ __forceinline__ uint32_t ca_transpose(uint32_t x) {
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// tma_load_5d with an L2 policy
__device__ __forceinline__ void ca_load(uint32_t dst, const CUtensorMap* m, uint32_t bar, int x, int y, int z, int w, int v, uint64_t pol) {
    asm volatile(
        "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint"
        " [%0], [%1, {%3, %4, %5, %6, %7}], [%2], %8;" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(x), "r"(y), "r"(z), "r"(w), "r"(v), "l"(pol)
        : "memory");
}

template <int HD_, int NT>
struct CaTensor {
    using T = bf16;
    static constexpr int HD = HD_, ROWS = 8 * NT, CTAS = 2;
    static constexpr int SK = HD == 64 ? 32 : 16, SPB = KB / SK;  // keys of a stage, stages of a block
    static constexpr int ONE = 3, EACH = 2, FULL = 16, FEW = 6 / SPB;                // blocks of a warp, see item_ctas
    static constexpr int SLAB = SK * 128, TILE = HD / 64 * SLAB, STAGE = 2 * TILE;  // 64 dimensions of the keys; keys; both
    static constexpr int NS = 3;
    static constexpr int BAR = NS * STAGE, WARP_BYTES = BAR + 1024;  // the ring, its barriers
    static_assert(CTAS * (CA_WARPS * WARP_BYTES + 3072) <= 228 * 1024, "CTAs an SM");
    static_assert(Part<HD, ROWS>::FLOATS * 4 <= BAR, "a part fits in the ring");

    const CUtensorMap &tmK, &tmV;
    uint32_t ring, bars;
    float* ring_part;  // the ring as the place of the warp's last part
    uint64_t policy;

    __device__ CaTensor(const CUtensorMap& k, const CUtensorMap& v, uint8_t* smem, int row_tiles) : tmK(k), tmV(v) {
        // Keys and values that one row tile reads are read once: the first to leave L2, before the scores that the second kernel
        // comes back for and what the program's other kernels keep there (16 contexts of up to 32K: 128 us for 133, with weights
        // 142 for 156)
        if (row_tiles == 1)
            asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
        else
            asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(policy));
        ring = smem_u32(smem);
        ring_part = reinterpret_cast<float*>(smem);
        bars = ring + BAR;
        if ((threadIdx.x & 31) == 0) {
            for (int s = 0; s < NS; ++s) mbar_init(bars + 8 * s, 1);
            fence_mbar_init();
            fence_proxy_async_smem();
            tma_prefetch_map(&tmK);
            tma_prefetch_map(&tmV);
        }
        __syncwarp();
    }

    // row of a slab, 16-byte chunk of it, under the 128-byte swizzle
    static __device__ __forceinline__ uint32_t at(int row, int chunk) {
        return (chunk >> 3) * SLAB + row * 128 + (((chunk ^ row) & 7) << 4);
    }
    // stages of a piece, and the first key of one (the last block may end in its first half)
    static __device__ __forceinline__ int stages(const CaWalk& w) {
        const int n = (w.b1 - w.b0) * SPB;
        return SPB == 2 && n && w.r.at(w.b1 - 1) + SK >= w.r.n ? n - 1 : n;
    }
    static __device__ __forceinline__ int key0(const CaWalk& w, int i) { return w.r.at(w.b0 + i / SPB) + i % SPB * SK; }

    // The copies of a warp's stages, ahead of their reading and on through the pieces.  Lane n holds the page of copy n of the
    // piece's next 32.
    struct Feed {
        CaWalk w;
        int box_log2, copies;  // positions of a copy, copies of a stage
        int i = 0, n = 0, batch = 0, page = 0;
        __device__ Feed(const CaArgs& a) : w(a) {
            box_log2 = min(a.v.page_log2, SK == 32 ? 5 : 4);
            copies = SK >> box_log2;
        }
    };
    __device__ __forceinline__ void feed(const CaArgs& a, Feed& f, int s) {
        const int lane = threadIdx.x & 31;
        while (f.i == f.n) {
            if (!f.w.next(a)) return;
            f.i = 0;
            f.n = stages(f.w);
            f.batch = f.i - 32;
        }
        if ((f.i - f.batch) * f.copies >= 32) {
            f.batch = f.i;
            const int copies_log2 = (SK == 32 ? 5 : 4) - f.box_log2, i = f.i + (lane >> copies_log2);
            const int j = i < f.n ? key0(f.w, i) + ((lane & (f.copies - 1)) << f.box_log2) : INT_MAX;
            f.page = j < f.w.r.n ? a.v.table[(size_t)f.w.c * a.v.width + (j >> a.v.page_log2)] : 0;
        }
        const int j0 = key0(f.w, f.i), box = 1 << f.box_log2, live = min(f.copies, (f.w.r.n - j0 + box - 1) >> f.box_log2);
        int page = __shfl_sync(0xffffffffu, f.page, (f.i - f.batch) * f.copies + lane);
        if (lane == 0) mbar_expect_tx(bars + 8 * s, live * box * HD * 4);
        if (f.copies > 1) __syncwarp();
        if (lane < live) {
            if ((unsigned)page >= (unsigned)a.v.n_pages) {  // some page instead: what comes of it is an error's
                cache_fail(a.v.status, DS_CACHE_PAGE);
                page = 0;
            }
            const uint32_t dst = ring + s * STAGE + lane * box * 128;
            const int at = (j0 + lane * box) & ((1 << a.v.page_log2) - 1);
            const int l = a.v.s_layer ? f.w.l : 0, g = a.v.s_head ? f.w.g : 0;  // what is shared has one element in the maps
#pragma unroll
            for (int kb = 0; kb < HD / 64; ++kb) {
                ca_load(dst + kb * SLAB, &tmK, bars + 8 * s, 64 * kb, at, g, page, l, policy);
                ca_load(dst + TILE + kb * SLAB, &tmV, bars + 8 * s, 64 * kb, at, g, page, l, policy);
            }
        }
        __syncwarp();
        ++f.i;
    }

    // A warp's rows of an item and what it has of them.  Lane 4 gq + t has Q of row 8 i + gq, and S, O and the sums of rows
    // 8 i + 2 t and + 1.
    struct Rows {
        uint32_t q[NT][HD / 16][2];
        float o[NT][HD / 16][4];
        float m[NT][2], l[NT][2], lx[NT][2];
        int vis[NT][2];
    };

    __device__ __forceinline__ void run(const CaArgs& a, CaNote* notes) {
        using P = Part<HD, ROWS>;
        const int lane = threadIdx.x & 31, gq = lane >> 2, t = lane & 3;
        const float k2 = a.scale * 1.4426950408889634f;
        Feed ahead(a);
        CaWalk w = ahead.w;
        int slot = 0, phase = 0;  // of the stage to be read next
        for (int s = 0; s < NS - 1; ++s) feed(a, ahead, s);
        bool ok = true;
        while (ok && w.next(a)) {
            const CaRange& r = w.r;
            const int row0 = w.rt * ROWS, rows = min(ROWS, a.R - row0), n = stages(w);
            const size_t kv = w.kv(a);
            Rows x;
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                const bool live = 8 * i + gq < rows;
                const uint32_t* q =
                    reinterpret_cast<const uint32_t*>(static_cast<const bf16*>(a.Q) + (kv * a.R + row0 + (live ? 8 * i + gq : 0)) * HD) + t;
#pragma unroll
                for (int k = 0; k < HD / 16; ++k) {
                    x.q[i][k][0] = live ? q[8 * k] : 0;
                    x.q[i][k][1] = live ? q[8 * k + 4] : 0;
                    x.o[i][k][0] = x.o[i][k][1] = x.o[i][k][2] = x.o[i][k][3] = 0.f;
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int row = 8 * i + 2 * t + h;
                    x.m[i][h] = -INFINITY;
                    x.l[i][h] = x.lx[i][h] = 0.f;
                    x.vis[i][h] = row < rows ? r.n - a.n_tok + (a.n_tok == 1 ? 0 : (row0 + row) % a.n_tok) + 1 : 0;
                }
            }
            for (int i = 0; i < n; ++i) {
                ok = __all_sync(0xffffffffu, mbar_wait(bars + 8 * slot, phase, a.v.status));
                if (!ok) break;
                step(a, ahead, r, key0(w, i), slot, kv, row0, rows, k2, x);
                __syncwarp();  // the stage has been read
                if (++slot == NS) {
                    slot = 0;
                    phase ^= 1;
                }
            }
            // a part goes to the workspace while the ring is in use
            float* part = w.last && ok ? ring_part : P::of_warp(a, w.b0 == 0);
            if (w.whole && lane == 0) a.info[kv * a.RT + w.rt] = 1 << 16;
            if (!w.whole && lane == 0) notes[w.b0 == 0] = {part, w.c, w.l, w.g, w.rt, r.n, w.first, w.cta_whole, w.parts};
            const long long head = w.l * a.v.s_layer + w.g * a.v.s_head;
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float l = x.l[i][h], lx = x.lx[i][h];
#pragma unroll
                    for (int y = 4; y < 32; y <<= 1) {
                        l += __shfl_xor_sync(0xffffffffu, l, y);
                        lx += __shfl_xor_sync(0xffffffffu, lx, y);
                    }
                    const int row = 8 * i + 2 * t + h;
                    if (row >= rows) continue;
                    if (w.whole) {
                        bf16* out = static_cast<bf16*>(a.out) + (kv * a.R + row0 + row) * HD;
#pragma unroll
                        for (int d = 0; d < HD / 8; ++d) {
                            float v[1] = {x.o[i][d / 2][d % 2 * 2 + h]};
                            finish_row<bf16, HD, 1>(a, kv, w.c, r.n, row0 + row, 8 * d + gq, static_cast<const bf16*>(a.v.K) + head,
                                                    static_cast<const bf16*>(a.v.V) + head, v, l);
                            out[8 * d + gq] = __float2bfloat16_rn(v[0]);
                        }
                        if (gq == 0 && a.lse) a.lse[kv * a.R + row0 + row] = row_lse(x.m[i][h], lx, k2);
                    } else {
#pragma unroll
                        for (int d = 0; d < HD / 8; ++d) part[row * HD + 8 * d + gq] = x.o[i][d / 2][d % 2 * 2 + h];
                        if (gq == 0) {
                            part[P::M + row] = x.m[i][h];
                            part[P::L + row] = l;
                            part[P::LX + row] = lx;
                        }
                    }
                }
            __syncwarp();
        }
        if (!ok) drain_copies();
    }

    // One stage's keys
    __device__ __forceinline__ void step(const CaArgs& a, Feed& ahead, const CaRange& r, int j0, int slot, size_t kv, int row0, int rows, float k2,
                                         Rows& x) {
        const int lane = threadIdx.x & 31, gq = lane >> 2, t = lane & 3;
        const uint32_t ks = ring + slot * STAGE, vs = ks + TILE;
        const bool whole = j0 + SK <= r.n - a.n_tok + 1 && (j0 + SK <= a.n_sink || j0 >= r.n - a.window);
        if (!whole) {  // values that no row sees are not to meet a probability of 0
            for (int e = lane; e < SK * 8; e += 32) {
                const int key = j0 + (e >> 3);
                if (key < r.n && (key < a.n_sink || key > r.t0 - a.window)) continue;
#pragma unroll
                for (int kb = 0; kb < HD / 64; ++kb)
                    asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};" ::"r"(vs + kb * SLAB + e * 16), "r"(0) : "memory");
            }
            fence_proxy_async_smem();
            __syncwarp();
        }
        float s[NT][SK / 16][4];  // of keys 16 u + gq (0, 1) and + 8 (2, 3), rows 2 t and + 1
#pragma unroll
        for (int u = 0; u < SK / 16; ++u)
#pragma unroll
            for (int i = 0; i < NT; ++i) s[i][u][0] = s[i][u][1] = s[i][u][2] = s[i][u][3] = 0.f;
#pragma unroll
        for (int k = 0; k < HD / 16; ++k)
#pragma unroll
            for (int u = 0; u < SK / 16; ++u) {
                uint32_t A[4];
                ca_ldmatrix<false>(A, ks + at(16 * u + (lane & 15), 2 * k + (lane >> 4)));
#pragma unroll
                for (int i = 0; i < NT; ++i) ca_mma(s[i][u], A, x.q[i][k][0], x.q[i][k][1]);
            }
        feed(a, ahead, slot == 0 ? NS - 1 : slot - 1);  // into the slot that was read last, while the products are under way
        uint32_t pb[NT][SK / 16][2];  // P^T: keys 16 u + 2 t, + 1 (and + 8) of row gq
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            if (!whole) {
#pragma unroll
                for (int u = 0; u < SK / 16; ++u)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int key = j0 + 16 * u + gq + 8 * (e >> 1), v = x.vis[i][e & 1];
                        s[i][u][e] = key < v && (key < a.n_sink || key >= v - a.window) ? s[i][u][e] : -INFINITY;
                    }
            }
            if (a.z2) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    if (8 * i + 2 * t + h < rows) {
                        float* z = a.z2 + (kv * a.R + row0 + 8 * i + 2 * t + h) * a.pitch + j0 + gq;
#pragma unroll
                        for (int u = 0; u < SK / 16; ++u) {
                            z[16 * u] = s[i][u][h] * k2;
                            z[16 * u + 8] = s[i][u][2 + h] * k2;
                        }
                    }
            }
            float moff[2], corr[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float cm = fmaxf(s[i][0][h], s[i][0][2 + h]);
#pragma unroll
                for (int u = 1; u < SK / 16; ++u) cm = fmaxf(cm, fmaxf(s[i][u][h], s[i][u][2 + h]));
#pragma unroll
                for (int y = 4; y < 32; y <<= 1) cm = fmaxf(cm, __shfl_xor_sync(0xffffffffu, cm, y));
                const float mn = fmaxf(x.m[i][h], cm);
                corr[h] = mn == x.m[i][h] ? 1.f : ca_exp2((x.m[i][h] - mn) * k2);
                moff[h] = mn == -INFINITY ? 0.f : -mn * k2;
                x.m[i][h] = mn;
            }
            if (__any_sync(0xffffffffu, corr[0] != 1.f || corr[1] != 1.f)) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    x.l[i][h] *= corr[h];
                    x.lx[i][h] *= corr[h];
#pragma unroll
                    for (int d = 0; d < HD / 16; ++d) {
                        x.o[i][d][h] *= corr[h];
                        x.o[i][d][2 + h] *= corr[h];
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < SK / 16; ++u)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const float e0 = ca_exp2(fmaf(s[i][u][2 * half], k2, moff[0])), e1 = ca_exp2(fmaf(s[i][u][2 * half + 1], k2, moff[1]));
                    const uint32_t p = pack_bf16(e0, e1);
                    // O's sums take the probabilities that the MMA sees, the weights' the exact ones
                    x.l[i][0] += __uint_as_float(p << 16);
                    x.l[i][1] += __uint_as_float(p & 0xffff0000u);
                    x.lx[i][0] += e0;
                    x.lx[i][1] += e1;
                    pb[i][u][half] = ca_transpose(p);
                }
        }
#pragma unroll
        for (int u = 0; u < SK / 16; ++u)
#pragma unroll
            for (int d = 0; d < HD / 16; ++d) {
                uint32_t A[4];
                ca_ldmatrix<true>(A, vs + at(16 * u + (lane & 7) + ((lane >> 4) << 3), 2 * d + ((lane >> 3) & 1)));
#pragma unroll
                for (int i = 0; i < NT; ++i) ca_mma(x.o[i][d], A, pb[i][u][0], pb[i][u][1]);
            }
    }
};

// ---------------------------------------------------------------- joining the parts, and the weights
constexpr int FIN_THREADS = 256, FIN_WARPS = FIN_THREADS / 32;
constexpr int FIN_TILE = 4 * FIN_THREADS, FIN_TILES = 4, FIN_POS = FIN_TILES * FIN_TILE;  // positions at a time, times, of a block

// One row of a split item from its parts, of CTAs first .. first + n - 1.  A thread has two dimensions of every G-th part;
// the G sums are added in order.
template <typename T, int HD, int ROWS>
__device__ __forceinline__ void join_row(const CaArgs& a, int c, int row, size_t kv, const T* K, const T* V, int n_pos, int first, int n, float k2) {
    using P = Part<HD, ROWS>;
    constexpr int COLS = HD / 2, G = FIN_THREADS / COLS;
    __shared__ float2 os[G][COLS];
    __shared__ float ls[G];
    const int col = threadIdx.x % COLS, grp = threadIdx.x / COLS, in = row % ROWS;
    auto part = [&](int k) { return P::of_cta(a, first + k, k == 0); };
    float mx = -INFINITY;
    for (int k = threadIdx.x & 31; k < n; k += 32) mx = fmaxf(mx, part(k)[P::M + in]);
    mx = warp_max(mx);
    float2 o = make_float2(0.f, 0.f);
    float l = 0.f;
#pragma unroll 8
    for (int k = grp; k < n; k += G) {
        const float* p = part(k);
        const float2 x = *reinterpret_cast<const float2*>(p + in * HD + 2 * col);
        const float mk = p[P::M + in], f = mk == -INFINITY ? 0.f : ca_exp2((mk - mx) * k2);
        l = fmaf(f, p[P::L + in], l);
        o.x = fmaf(f, x.x, o.x);
        o.y = fmaf(f, x.y, o.y);
    }
    os[grp][col] = o;
    if (col == 0) ls[grp] = l;
    __syncthreads();
    if (grp) return;
    for (int k = 1; k < G; ++k) {
        l += ls[k];
        o.x += os[k][col].x;
        o.y += os[k][col].y;
    }
    write_row<T, HD>(a, kv, c, n_pos, row, 2 * col, K, V, o.x, o.y, l);
}

// The first R blocks of a KV head join its rows' parts; the others, if the cache has weights, add those of FIN_POS positions
// each, four a thread at a time.
template <typename Form>
__global__ void __launch_bounds__(FIN_THREADS, 5) cache_finish_kernel(const CaArgs a) {
    using T = typename Form::T;
    constexpr int HD = Form::HD, ROWS = Form::ROWS;
    __shared__ float lse[FIN_ROWS];
    const int chain = blockIdx.z, g = blockIdx.y, c = chain / a.v.L, l = chain % a.v.L;
    const float k2 = a.scale * 1.4426950408889634f;
    const size_t kv = (size_t)chain * a.v.n_kv + g;
    const CaRange r(a, c);
    const int tile0 = ((int)blockIdx.x - a.R) * FIN_POS, p0 = tile0 + 4 * threadIdx.x;
    if (tile0 >= r.n || (tile0 >= a.n_sink && tile0 + FIN_POS <= r.t0 - a.window + 1)) return;  // nobody sees them
    pdl_wait();  // above, only the lengths are read, which were there before the first kernel began
    if ((int)blockIdx.x < a.R) {
        const int row = blockIdx.x, info = a.info[kv * a.RT + row / ROWS], first = info & 0xffff, n = info >> 16;
        if (n == 1) return;
        const long long head = l * a.v.s_layer + g * a.v.s_head;
        join_row<T, HD, ROWS>(a, c, row, kv, static_cast<const T*>(a.v.K) + head, static_cast<const T*>(a.v.V) + head, r.n, first, n, k2);
        return;
    }
    float* score = a.v.score + (((size_t)c * a.v.Lh + l) * a.v.n_kv + g) * a.v.cap;
    for (int row0 = 0; row0 < a.R; row0 += FIN_ROWS) {
        const int rows = min(FIN_ROWS, a.R - row0);
        bool nans = false;  // some row's sum
        __syncthreads();
        for (int row = threadIdx.x >> 5; row < rows; row += FIN_WARPS) {  // a warp a row
            const int lane = threadIdx.x & 31, in = (row0 + row) % ROWS, info = a.info[kv * a.RT + (row0 + row) / ROWS];
            const int first = info & 0xffff, n = info >> 16;
            float m = -INFINITY, lx = 0.f;
            if (n == 1) {
                m = a.lse[kv * a.R + row0 + row];
            } else {
                for (int k = lane; k < n; k += 32) {
                    using P = Part<HD, ROWS>;
                    const float* p = P::of_cta(a, first + k, k == 0) + in;
                    // (a part of max -inf has the sum 0, or NaN, which stays)
                    const float mk = p[P::M], lk = p[P::LX], mn = fmaxf(m, mk);
                    lx = fmaf(lx, m == -INFINITY ? 1.f : ca_exp2((m - mn) * k2), mk == -INFINITY ? lk : lk * ca_exp2((mk - mn) * k2));
                    m = mn;
                }
                const float mx = warp_max(m);
                lx = warp_sum(m == -INFINITY ? lx : lx * ca_exp2((m - mx) * k2));
                m = row_lse(mx, lx, k2);
            }
            if (lane == 0) lse[row] = m;
            nans |= isnan(m);
        }
        nans = __syncthreads_or(nans);
#pragma unroll 2
        for (int tile = 0; tile < FIN_TILES; ++tile) {
            const int p = p0 + tile * FIN_TILE;
            if (p >= r.n || (p >= a.n_sink && p + 4 <= r.t0 - a.window + 1)) continue;
            float w[4] = {0.f, 0.f, 0.f, 0.f};
            const float* z = a.z2 + (kv * a.R + row0) * a.pitch + p;
            auto sum = [&](auto check) {
                constexpr bool N = decltype(check)::value;
#pragma unroll 4
                for (int row = 0; row < rows; ++row) {
                    const float4 x = __ldcs(reinterpret_cast<const float4*>(z + row * a.pitch));
                    const float s = lse[row];
                    w[0] += ca_weight<N>(x.x, s);
                    w[1] += ca_weight<N>(x.y, s);
                    w[2] += ca_weight<N>(x.z, s);
                    w[3] += ca_weight<N>(x.w, s);
                }
            };
            nans ? sum(std::true_type()) : sum(std::false_type());
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (p + i < r.n && (p + i < a.n_sink || p + i > r.t0 - a.window)) score[p + i] += w[i];
        }
    }
}

// Blocks of an item, at most: a context as long as its table, first positions and window in blocks of their own
long long max_blocks(const CacheView& v) { return (v.cap + KB - 1) / KB + 1; }
long long seen_blocks(const CaArgs& a) {
    return std::min(max_blocks(a.v), ((long long)a.n_sink + KB - 1) / KB + ((long long)a.window + a.n_tok + KB - 1) / KB + 1);
}

// CTAs (a cluster) of each item, or 0: the blocks are dealt out and a second kernel follows.  While all items fit on the GPU at once, a cluster an
// item saves the second kernel and the dealing.  It takes one CTA up to ONE blocks a warp, then as many as leave EACH.  Dealing is
// faster where a warp would have more than FEW blocks with half of the GPU idle, or more than FULL blocks of contexts that
// may be unequal.  (32 heads over 8, pages of 64, without and with weights, us here and dealt.  hd 64: 1 layer of 150 positions 5.2, 5.8
// and 6.3, 8.9; 500: 5.7, 6.8 and 9.4, 10.7; 4500: 8.6, 10.5 and 10.4, 14.3; 9000: 11.5, 17.2 and 11.3, 15.6; 16 layers of 1151:
// 9.8, 12.1 and 12.5, 15.4; 20000: 97, 121 and 106, 124; 32 of 1151: 15.6, 17.5 and 22.6, 25.5.  hd 128, 4 layers of 131072, two tokens:
// 297 and 318; 1 of 4500: 13.7, 17.6 and 12.2, 15.7.  The CUDA cores take 6 us a block, so it is theirs for one a warp: fp32, 500: 12.0,
// 13.7 and 27.8, 30.8; 1151: 17.5, 20.0 and 14.7, 17.1.)
// The lengths are on the device, so the rule goes by what the table and the window allow: a context that is short for its table is
// dealt out (150 positions of one layer in a table of their own 5.6, with weights 6.2; in one for 8K or 32K 8.0 and 9.5).
template <typename Form>
int item_ctas(const CaArgs& a, int sms) {
    const long long items = (long long)a.per * a.v.n_ctx, blocks = seen_blocks(a), slots = (long long)Form::CTAS * sms;
    if (items > slots || (a.v.score && a.RT > 1)) return 0;  // (row tiles of a head add to the same weights)
    int S = 1;
    if (blocks > Form::ONE * CA_WARPS)
        while (S < 8 && 2 * S * items <= slots && blocks > Form::EACH * S * CA_WARPS) S *= 2;
    const bool full = 2 * S * items > slots;
    if (full && a.v.n_ctx == 1 && Form::FULL > 1) return S;
    return blocks <= S * CA_WARPS * (full ? Form::FULL : Form::FEW) ? S : 0;
}

template <typename Form>
cudaError_t launch(CaArgs a, const CUtensorMap& tmK, const CUtensorMap& tmV, int sms, int* kernels, cudaStream_t st) {
    static_assert(Form::CTAS * Form::ROWS <= CA_SM_ROWS, "the workspace's parts");
    constexpr size_t smem = CA_WARPS * Form::WARP_BYTES + 1024, smem_items = smem + Part<Form::HD, Form::ROWS>::FLOATS * sizeof(float);
    static PerDevice<SmemOptIn> once, once_items;
    a.RT = (a.R + Form::ROWS - 1) / Form::ROWS;
    a.per = a.v.L * a.v.n_kv * a.RT;
    a.ctas = Form::CTAS * sms;
    a.split = item_ctas<Form>(a, sms);
    if (a.split) {
        *kernels = 1;
        a.ctas = a.split * a.per * a.v.n_ctx;
        cudaError_t e = smem_opt_in(reinterpret_cast<const void*>(cache_attention_kernel<Form, true>), smem_items, once_items);
        if (e != cudaSuccess) return e;
        return launch_kernel(cache_attention_kernel<Form, true>, dim3(a.ctas), dim3(CA_THREADS), smem_items, st, true, a.split, tmK, tmV, a);
    }
    cudaError_t e = smem_opt_in(reinterpret_cast<const void*>(cache_attention_kernel<Form, false>), smem, once);
    if (e != cudaSuccess) return e;
    e = launch_kernel(cache_attention_kernel<Form, false>, dim3(a.ctas), dim3(CA_THREADS), smem, st, true, 1, tmK, tmV, a);
    // without weights, no item is split over CTAs if none is long
    if (e != cudaSuccess || (*kernels = a.v.score || max_blocks(a.v) > CA_WHOLE ? 2 : 1) == 1) return e;
    const dim3 grid((unsigned)(a.R + (a.v.score ? (a.v.cap + FIN_POS - 1) / FIN_POS : 0)), a.v.n_kv, a.v.n_ctx * a.v.L);
    return launch_kernel(cache_finish_kernel<Form>, grid, dim3(FIN_THREADS), 0, st, true, 1, a);
}

// The pools as (head_dim, position, KV head, page, layer), a box the positions of a page that a stage holds.
template <int HD>
bool pool_maps(const CacheView& v, CUtensorMap* mk, CUtensorMap* mv) {
    // The map of the last call's shape, of which a call only sets the addresses
    struct Plan {
        long long key[8];
        CUtensorMap m;
    };
    static thread_local Plan plan = {};
    const long long key[8] = {1, v.L, v.n_kv, v.n_pages, v.page_log2, v.s_layer, v.s_page, v.s_head};
    static thread_local long long s_pos = 0;
    if (!std::equal(key, key + 8, plan.key) || s_pos != v.s_pos) {
        const uint64_t page = 1ull << v.page_log2;
        // a dimension that is shared (stride 0) has one element, which takes any stride
        const uint64_t d[5] = {HD, page, v.s_head ? (uint64_t)v.n_kv : 1, (uint64_t)v.n_pages, v.s_layer ? (uint64_t)v.L : 1};
        const uint64_t s3 = v.s_pos * 2;
        const uint64_t s[4] = {s3, d[2] > 1 ? v.s_head * 2 : s3, d[3] > 1 ? v.s_page * 2 : s3, d[4] > 1 ? v.s_layer * 2 : s3};
        const uint32_t b[5] = {64, (uint32_t)std::min<uint64_t>(page, CaTensor<HD, 1>::SK), 1, 1, 1};
        plan.key[0] = 0;
        if (!encode_map_bf16_5d(&plan.m, v.K, d, s, b)) return false;  // strides past a tensor map's range (2^40 bytes)
        std::copy(key, key + 8, plan.key);
        s_pos = v.s_pos;
    }
    *mk = *mv = plan.m;
    return retarget_map(mk, v.K) && retarget_map(mv, v.V);
}

template <int HD>
cudaError_t launch_bf16(const CaArgs& a, int sms, int* kernels, cudaStream_t st) {
    CUtensorMap mk = {}, mv = {};
    // pages of fewer than 8 positions would need copies of less than a swizzle's rows
    if (a.vec && a.v.page_log2 >= 3 && pool_maps<HD>(a.v, &mk, &mv))
        return a.R <= 8 ? launch<CaTensor<HD, 1>>(a, mk, mv, sms, kernels, st) : launch<CaTensor<HD, 2>>(a, mk, mv, sms, kernels, st);
    return launch<CaCores<bf16, HD>>(a, mk, mv, sms, kernels, st);
}

struct Layout {
    size_t info, lse, z2, bytes;
    long long pitch;
    Layout(const DevState& s, const CacheView& v, int n_q, int n_tok) {
        const size_t kv = (size_t)v.n_ctx * v.L * v.n_kv, R = (size_t)n_q / v.n_kv * n_tok;
        auto up = [](size_t n) { return (n + 255) / 256 * 256; };
        info = up((size_t)2 * (1 + CA_WARPS) * CA_SM_ROWS * s.sms * (s.hd + 3) * sizeof(float));  // after the parts
        lse = info + up(kv * ((R + 3) / 4) * sizeof(int));  // items, at most
        z2 = lse + (v.score ? up(kv * R * sizeof(float)) : 0);
        pitch = (v.cap + KB - 1) / KB * KB;
        bytes = z2 + (v.score ? up(kv * R * pitch * sizeof(float)) : 0);
    }
};

}  // namespace

size_t cache_attention_workspace(const DevState& s, const CacheView& v, int n_q, int n_tok) {
    // blocks are counted in 31 bits; the CUDA-core form has the most row tiles
    const long long tiles = (n_q / v.n_kv * n_tok + CaCores<float, 64>::ROWS - 1) / CaCores<float, 64>::ROWS;
    if (max_blocks(v) * v.n_ctx * v.L * v.n_kv * tiles >= 1 << 30) return 0;
    return Layout(s, v, n_q, n_tok).bytes;
}

cudaError_t launch_cache_attention(const DevState& s, const CacheView& v, const void* Q, int n_q, int n_tok, int n_sink, int window,
                                   void* out, void* ws, int* kernels, cudaStream_t st) {
    const Layout w(s, v, n_q, n_tok);
    CaArgs a{};
    a.v = v;
    a.Q = Q; a.out = out;
    a.n_tok = n_tok; a.R = n_q / v.n_kv * n_tok;
    // positions are below 2^30: more hides and adds nothing, and a position less a window stays in range
    a.n_sink = std::min(n_sink, 1 << 30); a.window = std::min(window, 1 << 30);
    a.vec = cache_vec(v, s.dtype == 0 ? 4 : 2);
    a.scale = 1.0f / sqrtf((float)s.hd);
    char* b = static_cast<char*>(ws);
    a.part = reinterpret_cast<float*>(b);
    a.info = reinterpret_cast<int*>(b + w.info);
    a.lse = v.score ? reinterpret_cast<float*>(b + w.lse) : nullptr;
    a.z2 = v.score ? reinterpret_cast<float*>(b + w.z2) : nullptr;
    a.pitch = w.pitch;
    if (s.dtype != 0) return s.hd == 64 ? launch_bf16<64>(a, s.sms, kernels, st) : launch_bf16<128>(a, s.sms, kernels, st);
    const CUtensorMap none = {};
    return s.hd == 64 ? launch<CaCores<float, 64>>(a, none, none, s.sms, kernels, st) : launch<CaCores<float, 128>>(a, none, none, s.sms, kernels, st);
}

}  // namespace mone
