// Attention of each context's newest tokens over its paged cache, and the weights that the cache's positions are given by it: what the
// forms over rows of the handle's type (cache_attention.cu) and over rows in 4 bits (cache4_attention.cu) share.
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
// Of a form IN_STEP the items are dealt out in groups, to as many CTAs each: heads of a layer, if they can, heads and layers.  Heads of a context, and
// row tiles of a head, are then read at the same positions at about the same time, so what they share (a sector of HBM where a position's heads
// lie beside one another, a tile's keys) is read once.
//
// For the weights the scores go to the workspace as well (4 bytes a row and position beside the 4 head_dim, in bf16, of its
// key and value), and the second kernel, or the cluster's end, adds exp(z - max) / sum over the rows of a KV head.
#pragma once

#include <algorithm>
#include <climits>
#include <cstddef>
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
    int groups;                // of items, each dealt out to ctas / groups CTAs: a context's items g, g + groups, .. are group g's
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
template <bool IN_STEP>
struct CaDeal {
    // items of a context and CTAs that are dealt out together
    static __device__ __forceinline__ int items(const CaArgs& a) { return IN_STEP ? udiv(a.per, a.groups) : a.per; }
    static __device__ __forceinline__ int ctas(const CaArgs& a) { return IN_STEP ? udiv(a.ctas, a.groups) : a.ctas; }
    int total, share, per;
    int units, mine, incl;  // of context c0 + lane, of those scanned last: units of an item, of its items, up to its last
    __device__ CaDeal(const CaArgs& a) : per(items(a)) {
        total = 0;
        for (int c0 = 0; c0 < a.v.n_ctx; c0 += 32) total = scan(a, c0, total);
        const int n = ctas(a);
        share = max(udiv(total + n - 1, n), CA_SHARE);
    }
    // with `before` units ahead of them; returns the units up to the last
    __device__ int scan(const CaArgs& a, int c0, int before) {
        const int lane = threadIdx.x & 31;
        units = c0 + lane < a.v.n_ctx ? CaRange(a, c0 + lane).units() : 0;
        mine = units * per;
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
    // the first unit of CTA w of them
    __device__ int start(const CaArgs& a, int w) {
        const int u = w * share;  // below 2^30 + ctas share
        if (u >= total) return total;
        int base, c;
        const int n = locate(a, u, base, c);
        return n <= CA_WHOLE ? base + udiv(u - base, n) * n : u;
    }
};

// The pieces of a warp, one after the other: blocks [b0, b1) of an item
template <bool IN_STEP>
struct alignas(16) CaWalk {
    using Deal = CaDeal<IN_STEP>;
    int u, end, ctx0, c, units;
    CaRange r;
    int l, g, rt, b0, b1;
    int share, parts;         // of a CTA; CTAs that have a part of the item
    bool whole, cta_whole;    // the warp has the item whole, the CTA has
    bool first, last;         // the item begins in the CTA's share; the warp's last piece
    int cta0, cta1;           // the CTA's units
    __device__ CaWalk() {}
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
        Deal deal(a);
        share = deal.share;
        // CTAs behind the last group's have no unit
        const int n = Deal::ctas(a), rank = IN_STEP ? blockIdx.x - min(udiv(blockIdx.x, n), a.groups - 1) * n : blockIdx.x;
        cta0 = deal.start(a, rank);
        cta1 = deal.start(a, rank + 1);
        share_out();
        if (u < end) {
            units = deal.locate(a, u, ctx0, c);
            r = CaRange(a, c);
        }
    }
    __device__ bool next(const CaArgs& a) {
        if (u >= end) return false;
        while (u - ctx0 >= units * Deal::items(a)) {
            ctx0 += units * Deal::items(a);
            r = CaRange(a, ++c);
            units = r.units();
        }
        int in_ctx = udiv(u - ctx0, units);
        b0 = u - ctx0 - in_ctx * units;
        if (IN_STEP && a.groups > 1) in_ctx = in_ctx * a.groups + udiv(blockIdx.x, Deal::ctas(a));
        const int lg = a.RT == 1 ? in_ctx : udiv(in_ctx, a.RT);
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

// What a form is, beside its kernel code: WARP_BYTES of shared memory a warp, the first ALIGN-ed; Args, a CaArgs with what else it takes;
// Maps, the tensor maps it takes; Head, the rows of a layer's KV head in the pools; T, the type of queries and outputs.
struct NoMaps {};

// Rows of type T_
template <typename T_>
struct DenseHead {
    const T_ *K, *V;
    long long s_page, s_pos;
    struct Row {
        const T_ *K, *V;
        __device__ float k(int d) const { return to_f<T_>(K[d]); }
        __device__ float v(int d) const { return to_f<T_>(V[d]); }
    };
    __device__ DenseHead(const CaArgs& a, int l, int g) : s_page(a.v.s_page), s_pos(a.v.s_pos) {
        const long long head = l * a.v.s_layer + g * a.v.s_head;
        K = static_cast<const T_*>(a.v.K) + head;
        V = static_cast<const T_*>(a.v.V) + head;
    }
    __device__ Row row(int page, int place) const {
        const long long off = page * s_page + place * s_pos;
        return {K + off, V + off};
    }
};

// A row of Q over the positions it sees and no others, by one thread: N dimensions from d0.  A block's products take a
// value row times a probability of 0 for the rows that do not see it, which is NaN where the value is not finite; only
// with several tokens do the rows of an item differ in what they see.  Reached by non-finite inputs only.
template <typename Form, int N>
__device__ __noinline__ void row_again(const typename Form::Args& a, const typename Form::T* q, int layer, int g, const int* table,
                                       int vis, int d0, float* o) {
    using T = typename Form::T;
    constexpr int HD = Form::HD;
    const typename Form::Head head(a, layer, g);
    float m = -INFINITY, l = 0.f;
    for (int d = 0; d < N; ++d) o[d] = 0.f;
    for (int j = a.n_sink > 0 ? 0 : max(0, vis - a.window); j < vis; ++j) {
        if (j >= a.n_sink && j < vis - a.window) j = vis - a.window;
        if (j >= vis) break;
        const int page = cache_page(a.v, table, j >> a.v.page_log2);
        if (page < 0) continue;
        const auto row = head.row(page, j & ((1 << a.v.page_log2) - 1));
        float z = 0.f;
        for (int d = 0; d < HD; ++d) z = fmaf(to_f<T>(q[d]), row.k(d), z);
        z *= a.scale;
        if (z == -INFINITY) continue;
        const float mn = fmaxf(m, z), corr = __expf(m - mn), p = __expf(z - mn);
        m = mn;
        l = fmaf(l, corr, p);
        for (int d = 0; d < N; ++d) o[d] = fmaf(o[d], corr, p * row.v(d0 + d));
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

// N dimensions from d of a row, from its O and sum, ready to be stored
template <typename Form, int N>
__device__ __forceinline__ void finish_row(const typename Form::Args& a, size_t kv, int c, int layer, int g, int n, int row, int d,
                                           float (&o)[N], float l) {
    const float inv = l == 0.f ? 0.f : 1.f / l;  // no key that counts: 0
    bool bad = false;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        o[i] *= inv;
        bad |= !isfinite(o[i]);
    }
    if (a.n_tok > 1 && bad) {
        float w[N];
        row_again<Form, N>(a, static_cast<const typename Form::T*>(a.Q) + (kv * a.R + row) * Form::HD, layer, g, a.v.table + (size_t)c * a.v.width,
                           n - a.n_tok + row % a.n_tok + 1, d, w);
#pragma unroll
        for (int i = 0; i < N; ++i) o[i] = w[i];
    }
}
template <typename Form>
__device__ __forceinline__ void write_row(const typename Form::Args& a, size_t kv, int c, int layer, int g, int n, int row, int d,
                                          float o0, float o1, float l) {
    using T = typename Form::T;
    float o[2] = {o0, o1};
    finish_row<Form, 2>(a, kv, c, layer, g, n, row, d, o, l);
    store2<T>(static_cast<T*>(a.out) + (kv * a.R + row) * Form::HD + d, o[0], o[1]);
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
__device__ __forceinline__ void cluster_end(const typename Form::Args& a, const CaNote* notes, float* mine) {
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
        auto write = [&](int row, int d, float o0, float o1, float sum) { write_row<Form>(a, kv, c, l, g, r.n, row0 + row, d, o0, o1, sum); };
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
cache_attention_kernel(const __grid_constant__ typename Form::Maps maps, const typename Form::Args a) {
    constexpr int HD = Form::HD, ROWS = Form::ROWS;
    using P = Part<HD, ROWS>;
    extern __shared__ uint8_t ca_raw[];
    __shared__ CaNote notes[2 * CA_WARPS];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(ca_raw) + Form::ALIGN - 1) & ~uintptr_t(Form::ALIGN - 1));
    const int warp = threadIdx.x >> 5;
    if ((threadIdx.x & 31) < 2) notes[2 * warp + (threadIdx.x & 31)].part = nullptr;
    __syncwarp();
    {
        Form form(maps, smem + warp * Form::WARP_BYTES, a.RT);
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
        if (threadIdx.x == 0 && it.first) a.info[kv * a.RT + it.rt] = blockIdx.x | it.parts << 16;
        float* to = it.whole ? nullptr : P::of_cta(a, blockIdx.x, it.first);
        for (int e = 2 * threadIdx.x; e < rows * HD; e += 2 * CA_THREADS) {
            const int row = e / HD, d = e - row * HD;
            const auto x = CaJoined::of<P>(ps, e, row, k2);
            if (to) {
                *reinterpret_cast<float2*>(to + e) = make_float2(x.o0, x.o1);
                if (d == 0) to[P::M + row] = x.mx, to[P::L + row] = x.l, to[P::LX + row] = x.lx;
            } else {
                write_row<Form>(a, kv, it.c, it.l, it.g, it.n, row0 + row, d, x.o0, x.o1, x.l);
                if (d == 0 && a.lse) a.lse[kv * a.R + row0 + row] = row_lse(x.mx, x.lx, k2);
            }
        }
    }
}

// an 8 x 8 matrix of 16-bit elements, two of a row a lane, transposed
__device__ __forceinline__ uint32_t ca_transpose(uint32_t x) {
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// ---------------------------------------------------------------- joining the parts, and the weights
constexpr int FIN_THREADS = 256, FIN_WARPS = FIN_THREADS / 32;
constexpr int FIN_TILE = 4 * FIN_THREADS, FIN_TILES = 4, FIN_POS = FIN_TILES * FIN_TILE;  // positions at a time, times, of a block

// One row of a split item from its parts, of CTAs first .. first + n - 1.  A thread has two dimensions of every G-th part;
// the G sums are added in order.
template <typename Form>
__device__ __forceinline__ void join_row(const typename Form::Args& a, int c, int layer, int g, int row, size_t kv, int n_pos,
                                         int first, int n, float k2) {
    constexpr int HD = Form::HD, ROWS = Form::ROWS;
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
    write_row<Form>(a, kv, c, layer, g, n_pos, row, 2 * col, o.x, o.y, l);
}

// The first R blocks of a KV head join its rows' parts; the others, if the cache has weights, add those of FIN_POS positions
// each, four a thread at a time.
template <typename Form>
__global__ void __launch_bounds__(FIN_THREADS, 5) cache_finish_kernel(const typename Form::Args a) {
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
        join_row<Form>(a, c, l, g, row, kv, r.n, first, n, k2);
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
inline long long max_blocks(const CacheView& v) { return (v.cap + KB - 1) / KB + 1; }
inline long long seen_blocks(const CaArgs& a) {
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
// (The 4-bit form has its own numbers, at its constants.)
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
    // Dealt out in groups, long items gain more from the CTAs that clusters would leave idle than the second kernel takes: from 8 blocks a warp times
    // the idle share on, or 10 and 20 with clusters of 4 and 2, whose more items take longer to join.  (4-bit rows, 32 heads over 8, hd 128, two
    // tokens, us in clusters and dealt: 5 layers, 8 a cluster, half idle, 8192 positions 21.1 and 20.9, 131072 189 and 137; 6 layers, 16384
    // 33.5 and 35.0, 32768 56.1 and 54.1; 16 layers, 4 a cluster, a sixth idle, 16384 69.8 and 72.4, 65536 239 and 222; fp32, 2 a cluster, nearly half
    // idle, 8192 53.3 and 56.5, 16384 97.1 and 90.5.  With one a cluster it could be sooner: 10 layers of 32 KV heads, nearly half idle, 4096 52.8 and 52.0, 8192 97
    // and 83, 16384 186 and 146; 15, a fifth idle, 4096 66 and 70, 8192 123 and 117, 16384 235 and 210.)
    const bool idle = Form::IN_STEP && (slots - S * items) * blocks >= (long long)std::max(8, 40 / S) * slots * S * CA_WARPS;
    if (full && a.v.n_ctx == 1 && Form::FULL > 1 && !idle) return S;
    return blocks <= S * CA_WARPS * (full ? Form::FULL : 3 * S * items > slots ? Form::SOME : Form::FEW) ? S : 0;
}

template <typename Form>
cudaError_t launch(typename Form::Args a, const typename Form::Maps& maps, int sms, int* kernels, cudaStream_t st) {
    static_assert(Form::CTAS * Form::ROWS <= CA_SM_ROWS, "the workspace's parts");
    constexpr size_t smem = CA_WARPS * Form::WARP_BYTES + Form::ALIGN, smem_items = smem + Part<Form::HD, Form::ROWS>::FLOATS * sizeof(float);
    static PerDevice<SmemOptIn> once, once_items;
    a.RT = (a.R + Form::ROWS - 1) / Form::ROWS;
    a.per = a.v.L * a.v.n_kv * a.RT;
    a.ctas = Form::CTAS * sms;
    a.split = item_ctas<Form>(a, sms);
    a.groups = 1;
    if (a.split) {
        *kernels = 1;
        a.ctas = a.split * a.per * a.v.n_ctx;
        cudaError_t e = smem_opt_in(reinterpret_cast<const void*>(cache_attention_kernel<Form, true>), smem_items, once_items);
        if (e != cudaSuccess) return e;
        return launch_kernel(cache_attention_kernel<Form, true>, dim3(a.ctas), dim3(CA_THREADS), smem_items, st, true, a.split, maps, a);
    }
    if (Form::IN_STEP) {  // the most groups, of all heads of one layer or more, that leave out at most a sixteenth of the CTAs
        const int heads = a.v.n_kv * a.RT, all = a.ctas;
        for (int k = a.v.L; k > 0 && a.groups == 1; --k) {
            const int groups = k * heads;
            if (a.v.L % k == 0 && 16 * (all / groups * groups) >= 15 * all) a.groups = groups;
        }
    }
    cudaError_t e = smem_opt_in(reinterpret_cast<const void*>(cache_attention_kernel<Form, false>), smem, once);
    if (e != cudaSuccess) return e;
    e = launch_kernel(cache_attention_kernel<Form, false>, dim3(a.ctas), dim3(CA_THREADS), smem, st, true, 1, maps, a);
    // without weights, no item is split over CTAs if none is long
    if (e != cudaSuccess || (*kernels = a.v.score || max_blocks(a.v) > CA_WHOLE ? 2 : 1) == 1) return e;
    const dim3 grid((unsigned)(a.R + (a.v.score ? (a.v.cap + FIN_POS - 1) / FIN_POS : 0)), a.v.n_kv, a.v.n_ctx * a.v.L);
    return launch_kernel(cache_finish_kernel<Form>, grid, dim3(FIN_THREADS), 0, st, true, 1, a);
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


// What every form's call has in common
inline void ca_common(CaArgs& a, const DevState& s, const CacheView& v, const Layout& w, const void* Q, int n_q, int n_tok, int n_sink,
                      int window, void* out, void* ws) {
    a.v = v;
    a.Q = Q; a.out = out;
    a.n_tok = n_tok; a.R = n_q / v.n_kv * n_tok;
    // positions are below 2^30: more hides and adds nothing, and a position less a window stays in range
    a.n_sink = std::min(n_sink, 1 << 30); a.window = std::min(window, 1 << 30);
    a.scale = 1.0f / sqrtf((float)s.hd);
    char* b = static_cast<char*>(ws);
    a.part = reinterpret_cast<float*>(b);
    a.info = reinterpret_cast<int*>(b + w.info);
    a.lse = v.score ? reinterpret_cast<float*>(b + w.lse) : nullptr;
    a.z2 = v.score ? reinterpret_cast<float*>(b + w.z2) : nullptr;
    a.pitch = w.pitch;
}

}  // namespace

}  // namespace mone
