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
__global__ void __launch_bounds__(CA_THREADS, Form::CTAS)
cache_attention_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const CaArgs a) {
    using T = typename Form::T;
    constexpr int HD = Form::HD, ROWS = Form::ROWS, PART = Form::WARP_BYTES / 4;
    extern __shared__ uint8_t ca_raw[];
    float* ca_smem = reinterpret_cast<float*>((reinterpret_cast<uintptr_t>(ca_raw) + 1023) & ~uintptr_t(1023));
    __shared__ int last;
    const CaShare sh(a);
    if (sh.begin >= sh.end) return;
    Form form(tmK, tmV, a, ca_smem + (threadIdx.x >> 5) * PART);
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
        form.piece(a, r, c, l, g, kv, row0, rows, Kp, Vp, b0, min(b1, r.nb), k2, ca_smem + (threadIdx.x >> 5) * PART);
        __syncthreads();
        auto mine = [&](int k, int i) { return ca_smem[k * PART + i]; };
        if (b0 == 0 && b1 == units) {
            finish_rows<T, HD, ROWS>(a, CA_WARPS, mine, nullptr, rows, k2, c, kv, row0, r, Kp, Vp);
        } else {
            // slot 1 of a CTA: the first part of an item, which the next CTAs go on with; slot 0: the part it begins with
            float* slot = a.part + (2ll * blockIdx.x + (b0 == 0)) * Part<HD, ROWS>::FLOATS;
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
                const float* p0 = a.part + 2ll * first * Part<HD, ROWS>::FLOATS;
                auto theirs = [&](int k, int i) { return __ldcg(p0 + (2ll * k + (k == 0)) * Part<HD, ROWS>::FLOATS + i); };
                finish_rows<T, HD, ROWS>(a, (int)parts, theirs, nullptr, rows, k2, c, kv, row0, r, Kp, Vp);
            }
        }
        __syncthreads();  // the warps' parts have been read
        u += b1 - b0;
    }
    form.done();
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
    static constexpr int WARP_BYTES = Part<HD, ROWS>::FLOATS * 4;

    __device__ CaCores(const CUtensorMap&, const CUtensorMap&, const CaArgs&, float*) {}
    __device__ void done() {}

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

    __device__ __forceinline__ void piece(const CaArgs& a, const CaRange& r, int c, int, int, size_t kv, int row0, int rows, const T* Kp,
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

// ---------------------------------------------------------------- tensor cores: bf16
// A block's keys and values come by TMA, whose box is the positions of a page in the block (a swizzled row of 64 dimensions
// each), into a ring that belongs to one warp: a lane looks up a page and starts its copies, the warp waits for the
// stage, and what it has read is free for the next copy without another warp's say.  16 rows (a row tile) are the M of
// m16n8k16: S = Q K^T by ldmatrix from the key rows, P from S's registers, O += P V by transposed ldmatrix.  A 128-row
// tcgen05 tile would be 1/32 full for the four heads that usually share a KV head; what bounds this kernel is the bytes.
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

template <int HD_>
struct CaTensor {
    using T = bf16;
    static constexpr int HD = HD_, ROWS = 16, CTAS = 2;
    static constexpr int SK = HD == 64 ? 32 : 16, SPB = KB / SK;  // keys of a stage, stages of a block
    static constexpr int SLAB = SK * 128, TILE = HD / 64 * SLAB, STAGE = 2 * TILE;  // 64 dimensions of the keys; keys; both
    static constexpr int NS = 3;
    static constexpr int BAR = NS * STAGE, WARP_BYTES = BAR + 1024;  // the ring (at a piece's end: its part), its barriers
    static_assert(Part<HD, ROWS>::FLOATS * 4 <= BAR, "a part fits in the ring");
    static_assert(CTAS * (CA_WARPS * WARP_BYTES + 2048) <= 228 * 1024, "CTAs an SM");

    const CUtensorMap &tmK, &tmV;
    uint32_t ring, bars;
    int slot = 0, phase = 0;   // of the stage to be read next
    bool ok = true;

    __device__ CaTensor(const CUtensorMap& k, const CUtensorMap& v, const CaArgs&, float* smem) : tmK(k), tmV(v) {
        ring = smem_u32(smem);
        bars = ring + BAR;
        if ((threadIdx.x & 31) == 0) {
            for (int s = 0; s < NS; ++s) mbar_init(bars + 8 * s, 1);
            fence_mbar_init();
            tma_prefetch_map(&tmK);
            tma_prefetch_map(&tmV);
        }
        __syncwarp();
    }
    __device__ void done() {
        if (!ok) drain_copies();
    }

    // row of a slab, 16-byte chunk of it, under the 128-byte swizzle
    static __device__ __forceinline__ uint32_t at(int row, int chunk) {
        return (chunk >> 3) * SLAB + row * 128 + (((chunk ^ row) & 7) << 4);
    }

    __device__ __forceinline__ void piece(const CaArgs& a, const CaRange& r, int c, int l, int g, size_t kv, int row0, int rows, const T*,
                                          const T*, int b0, int b1, float k2, float* part) {
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gq = lane >> 2, t = lane & 3;
        const int* table = a.v.table + (size_t)c * a.v.width;
        const int mask = (1 << a.v.page_log2) - 1, box = min(mask + 1, SK);  // positions that one copy brings
        const int cl = a.v.s_layer ? l : 0, cg = a.v.s_head ? g : 0;  // a dimension that is shared has one element in the maps
        const int first = b0 + warp, stages = first < b1 ? ((b1 - first + CA_WARPS - 1) / CA_WARPS) * SPB : 0;
        auto key0 = [&](int i) { return r.at(first + i / SPB * CA_WARPS) + i % SPB * SK; };
        auto issue = [&](int i, int s) {
            const int j = key0(i) + lane * box;
            const bool mine = lane * box < SK && j < r.n;
            const uint32_t who = __ballot_sync(0xffffffffu, mine);
            if (lane == 0) mbar_expect_tx(bars + 8 * s, __popc(who) * box * HD * 4);
            __syncwarp();
            if (mine) {
                const int page = max(0, cache_page(a.v, table, j >> a.v.page_log2));  // a wrong one is latched
                const uint32_t dst = ring + s * STAGE + lane * box * 128;
#pragma unroll
                for (int kb = 0; kb < HD / 64; ++kb) {
                    tma_load_5d(dst + kb * SLAB, &tmK, bars + 8 * s, 64 * kb, j & mask, cg, page, cl);
                    tma_load_5d(dst + TILE + kb * SLAB, &tmV, bars + 8 * s, 64 * kb, j & mask, cg, page, cl);
                }
            }
        };
        // rows gq and gq + 8 of the tile
        uint32_t qa[HD / 16][4];
        int vis[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int row = row0 + min(gq + 8 * h, rows - 1);
            const bool live = gq + 8 * h < rows;
            vis[h] = live ? r.n - a.n_tok + row % a.n_tok + 1 : 0;
            const uint32_t* q = reinterpret_cast<const uint32_t*>(static_cast<const bf16*>(a.Q) + (kv * a.R + row) * HD) + t;
#pragma unroll
            for (int k = 0; k < HD / 16; ++k) {
                qa[k][h] = live ? __ldg(q + 8 * k) : 0;
                qa[k][2 + h] = live ? __ldg(q + 8 * k + 4) : 0;
            }
        }
        float o[HD / 8][4], m[2] = {-INFINITY, -INFINITY}, lr[2] = {0.f, 0.f}, lx[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < HD / 8; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;
        // the part that the ring's bytes held before has been read: by everybody (the CTA's barrier), and for the copies
        fence_proxy_async_smem();
        __syncwarp();
        int ahead = 0;  // stages asked for; their slots follow `slot`
        for (int s = slot; ok && ahead < min(NS - 1, stages) && key0(ahead) < r.n; ++ahead) {
            issue(ahead, s);
            s = s + 1 == NS ? 0 : s + 1;
        }
        for (int i = 0; ok && i < stages && key0(i) < r.n; ++i) {
            if (ahead < stages && key0(ahead) < r.n) {  // into the slot that was read last
                int s = slot + NS - 1;
                issue(ahead++, s >= NS ? s - NS : s);
            }
            ok = __all_sync(0xffffffffu, mbar_wait(bars + 8 * slot, phase, a.v.status));
            if (!ok) break;
            const int j0 = key0(i);
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
            float s[SK / 8][4];
#pragma unroll
            for (int nt = 0; nt < SK / 8; ++nt) {
                s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.f;
#pragma unroll
                for (int k = 0; k < HD / 32; ++k) {
                    uint32_t b[4];
                    ca_ldmatrix<false>(b, ks + at(8 * nt + (lane & 7), 4 * k + (lane >> 3)));
                    ca_mma(s[nt], qa[2 * k], b[0], b[1]);
                    ca_mma(s[nt], qa[2 * k + 1], b[2], b[3]);
                }
            }
            if (!whole) {
#pragma unroll
                for (int nt = 0; nt < SK / 8; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int key = j0 + 8 * nt + 2 * t + (e & 1), h = e >> 1;
                        s[nt][e] = key < vis[h] && (key < a.n_sink || key >= vis[h] - a.window) ? s[nt][e] : -INFINITY;
                    }
            }
            if (a.z2) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    if (gq + 8 * h < rows) {
                        float* z = a.z2 + (kv * a.R + row0 + gq + 8 * h) * a.pitch + j0 + 2 * t;
#pragma unroll
                        for (int nt = 0; nt < SK / 8; ++nt)
                            *reinterpret_cast<float2*>(z + 8 * nt) = make_float2(s[nt][2 * h] * k2, s[nt][2 * h + 1] * k2);
                    }
            }
            float moff[2], corr[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float cm = fmaxf(s[0][2 * h], s[0][2 * h + 1]);
#pragma unroll
                for (int nt = 1; nt < SK / 8; ++nt) cm = fmaxf(cm, fmaxf(s[nt][2 * h], s[nt][2 * h + 1]));
                cm = fmaxf(cm, __shfl_xor_sync(0xffffffffu, cm, 1));
                cm = fmaxf(cm, __shfl_xor_sync(0xffffffffu, cm, 2));
                const float mn = fmaxf(m[h], cm);
                corr[h] = mn == m[h] ? 1.f : ca_exp2((m[h] - mn) * k2);
                moff[h] = mn == -INFINITY ? 0.f : -mn * k2;
                m[h] = mn;
            }
            if (__any_sync(0xffffffffu, corr[0] != 1.f || corr[1] != 1.f)) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    lr[h] *= corr[h];
                    lx[h] *= corr[h];
                }
#pragma unroll
                for (int j = 0; j < HD / 8; ++j) {
                    o[j][0] *= corr[0];
                    o[j][1] *= corr[0];
                    o[j][2] *= corr[1];
                    o[j][3] *= corr[1];
                }
            }
#pragma unroll
            for (int kk = 0; kk < SK / 16; ++kk) {
                uint32_t pa[4];  // rows gq, gq + 8 x keys (2 t, 2 t + 1), then the same of the next eight keys
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int nt = 2 * kk + (q >> 1), h = q & 1;
                    const float e0 = ca_exp2(fmaf(s[nt][2 * h], k2, moff[h])), e1 = ca_exp2(fmaf(s[nt][2 * h + 1], k2, moff[h]));
                    pa[q] = pack_bf16(e0, e1);
                    // O's sum takes the probabilities the MMA sees, the weights' the exact ones
                    lr[h] += __uint_as_float(pa[q] << 16) + __uint_as_float(pa[q] & 0xffff0000u);
                    lx[h] += e0 + e1;
                }
#pragma unroll
                for (int d = 0; d < HD / 16; ++d) {
                    uint32_t b[4];
                    ca_ldmatrix<true>(b, vs + at(16 * kk + (lane & 15), 2 * d + (lane >> 4)));
                    ca_mma(o[2 * d], pa, b[0], b[1]);
                    ca_mma(o[2 * d + 1], pa, b[2], b[3]);
                }
            }
            __syncwarp();  // the stage has been read
            if (++slot == NS) {
                slot = 0;
                phase ^= 1;
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int x = 1; x < 4; x <<= 1) {
                lr[h] += __shfl_xor_sync(0xffffffffu, lr[h], x);
                lx[h] += __shfl_xor_sync(0xffffffffu, lx[h], x);
            }
            const int row = gq + 8 * h;
            if (t == 0) {
                part[ROWS * HD + row] = m[h];
                part[ROWS * (HD + 1) + row] = lr[h];
                part[ROWS * (HD + 2) + row] = lx[h];
            }
            if (row < rows)
#pragma unroll
                for (int j = 0; j < HD / 8; ++j) *reinterpret_cast<float2*>(part + row * HD + 8 * j + 2 * t) = make_float2(o[j][2 * h], o[j][2 * h + 1]);
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
cudaError_t launch(CaArgs a, const CUtensorMap& tmK, const CUtensorMap& tmV, int sms, cudaStream_t st) {
    static_assert(Form::CTAS <= CA_CTAS, "the workspace holds the parts of CA_CTAS CTAs an SM");
    if (Form::CTAS * sms > kCacheCounters) return cudaErrorInvalidConfiguration;
    constexpr size_t smem = CA_WARPS * Form::WARP_BYTES + 1024;
    static PerDevice<SmemOptIn> once;
    cudaError_t e = smem_opt_in(reinterpret_cast<const void*>(cache_attention_kernel<Form>), smem, once);
    if (e != cudaSuccess) return e;
    a.RT = (a.R + Form::ROWS - 1) / Form::ROWS;
    a.per = (long long)a.v.L * a.v.n_kv * a.RT;
    cache_attention_kernel<Form><<<Form::CTAS * sms, CA_THREADS, smem, st>>>(tmK, tmV, a);
    if ((e = cudaGetLastError()) != cudaSuccess || !a.v.score) return e;
    const dim3 grid((unsigned)((a.v.cap + SC_POS - 1) / SC_POS), a.v.n_kv, a.v.n_ctx * a.v.L);
    cache_weights_kernel<<<grid, SC_THREADS, 0, st>>>(a);
    return cudaGetLastError();
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
        const uint32_t b[5] = {64, (uint32_t)std::min<uint64_t>(page, CaTensor<HD>::SK), 1, 1, 1};
        plan.key[0] = 0;
        if (!encode_map_bf16_5d(&plan.m, v.K, d, s, b)) return false;  // strides past a tensor map's range (2^40 bytes)
        std::copy(key, key + 8, plan.key);
        s_pos = v.s_pos;
    }
    *mk = *mv = plan.m;
    return retarget_map(mk, v.K) && retarget_map(mv, v.V);
}

template <int HD>
cudaError_t launch_bf16(const CaArgs& a, int sms, cudaStream_t st) {
    CUtensorMap mk = {}, mv = {};
    // pages of fewer than 8 positions would need copies of less than a swizzle's rows
    if (a.vec && a.v.page_log2 >= 3 && pool_maps<HD>(a.v, &mk, &mv)) return launch<CaTensor<HD>>(a, mk, mv, sms, st);
    return launch<CaCores<bf16, HD>>(a, mk, mv, sms, st);
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
    // positions are below 2^30: more hides and adds nothing, and a position less a window stays in range
    a.n_sink = std::min(n_sink, 1 << 30); a.window = std::min(window, 1 << 30);
    a.vec = cache_vec(v, s.dtype == 0 ? 4 : 2);
    a.scale = 1.0f / sqrtf((float)s.hd);
    char* b = static_cast<char*>(ws);
    a.count = reinterpret_cast<int*>(b);
    a.part = reinterpret_cast<float*>(b + w.part);
    a.lse = v.score ? reinterpret_cast<float*>(b + w.lse) : nullptr;
    a.z2 = v.score ? reinterpret_cast<float*>(b + w.z2) : nullptr;
    a.pitch = w.pitch;
    if (s.dtype != 0) return s.hd == 64 ? launch_bf16<64>(a, s.sms, st) : launch_bf16<128>(a, s.sms, st);
    const CUtensorMap none = {};
    return s.hd == 64 ? launch<CaCores<float, 64>>(a, none, none, s.sms, st) : launch<CaCores<float, 128>>(a, none, none, s.sms, st);
}

}  // namespace mone
