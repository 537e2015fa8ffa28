// Attention of each context's newest tokens over its paged cache (mone_cache_attention): the forms over rows of the handle's type.
#include "cache_attention.cuh"

namespace mone {

namespace {

// ---------------------------------------------------------------- CUDA cores: fp32, and rows that are not aligned
// Eight lanes share a key, each with head_dim / 8 of its dimensions; the four lane groups of a warp take every fourth key and
// keep a softmax of their own, joined at the end of the piece.
template <typename T_, int HD_>
struct CaCores {
    using T = T_;
    static constexpr int HD = HD_, ROWS = 4, CTAS = HD == 64 ? 3 : 2;
    static constexpr int VE = 16 / sizeof(T), D = HD / 8, NP = D / VE;  // elements of 16 bytes; dimensions and 16-byte pieces of a lane
    static constexpr int U = 2;                                         // keys of a lane group at a time
    static constexpr bool IN_STEP = false;
    using Walk = CaWalk<IN_STEP>;
    static constexpr int ONE = 1, EACH = 1, FULL = 1, SOME = 1, FEW = 1;          // blocks of a warp, see item_ctas
    static constexpr int WARP_BYTES = 2 * Part<HD, ROWS>::FLOATS * 4, ALIGN = 16;

    using Args = CaArgs;
    using Maps = NoMaps;
    using Head = DenseHead<T>;

    float* parts;

    __device__ CaCores(const NoMaps&, uint8_t* smem, int) : parts(reinterpret_cast<float*>(smem)) {}

    __device__ __forceinline__ void run(const CaArgs& a, CaNote* notes) {
        Walk walk(a);
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

    __device__ __forceinline__ void piece(const CaArgs& a, const Walk& walk, CaNote* notes) {
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
                    write_row<CaCores>(a, kv, c, walk.l, walk.g, r.n, row0 + i, dim, x[0], x[1], l[i]);
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
// tma_load_5d with an L2 policy
__device__ __forceinline__ void ca_load(uint32_t dst, const CUtensorMap* m, uint32_t bar, int x, int y, int z, int w, int v, uint64_t pol) {
    asm volatile(
        "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint"
        " [%0], [%1, {%3, %4, %5, %6, %7}], [%2], %8;" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(x), "r"(y), "r"(z), "r"(w), "r"(v), "l"(pol)
        : "memory");
}

struct PoolMaps {
    CUtensorMap K, V;
};

template <int HD_, int NT>
struct CaTensor {
    using T = bf16;
    static constexpr int HD = HD_, ROWS = 8 * NT, CTAS = 2;
    static constexpr int SK = HD == 64 ? 32 : 16, SPB = KB / SK;  // keys of a stage, stages of a block
    static constexpr bool IN_STEP = false;
    using Walk = CaWalk<IN_STEP>;
    static constexpr int ONE = 3, EACH = 2, FULL = 16, SOME = 6 / SPB, FEW = 6 / SPB;                // blocks of a warp, see item_ctas
    static constexpr int SLAB = SK * 128, TILE = HD / 64 * SLAB, STAGE = 2 * TILE;  // 64 dimensions of the keys; keys; both
    static constexpr int NS = 3;
    static constexpr int BAR = NS * STAGE, WARP_BYTES = BAR + 1024, ALIGN = 1024;  // the ring, its barriers
    static_assert(CTAS * (CA_WARPS * WARP_BYTES + 3072) <= 228 * 1024, "CTAs an SM");
    static_assert(Part<HD, ROWS>::FLOATS * 4 <= BAR, "a part fits in the ring");

    using Args = CaArgs;
    using Maps = PoolMaps;
    using Head = DenseHead<T>;

    const CUtensorMap &tmK, &tmV;
    uint32_t ring, bars;
    float* ring_part;  // the ring as the place of the warp's last part
    uint64_t policy;

    __device__ CaTensor(const PoolMaps& m, uint8_t* smem, int row_tiles) : tmK(m.K), tmV(m.V) {
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
    static __device__ __forceinline__ int stages(const Walk& w) {
        const int n = (w.b1 - w.b0) * SPB;
        return SPB == 2 && n && w.r.at(w.b1 - 1) + SK >= w.r.n ? n - 1 : n;
    }
    static __device__ __forceinline__ int key0(const Walk& w, int i) { return w.r.at(w.b0 + i / SPB) + i % SPB * SK; }

    // The copies of a warp's stages, ahead of their reading and on through the pieces.  Lane n holds the page of copy n of the
    // piece's next 32.
    struct Feed {
        Walk w;
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
        Walk w = ahead.w;
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
                            finish_row<CaTensor, 1>(a, kv, w.c, w.l, w.g, r.n, row0 + row, 8 * d + gq, v, l);
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

// The pools as (head_dim, position, KV head, page, layer), a box the positions of a page that a stage holds.
template <int HD>
bool pool_maps(const CacheView& v, PoolMaps* to) {
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
    to->K = to->V = plan.m;
    return retarget_map(&to->K, v.K) && retarget_map(&to->V, v.V);
}

template <int HD>
cudaError_t launch_bf16(const CaArgs& a, int sms, int* kernels, cudaStream_t st) {
    PoolMaps maps = {};
    // pages of fewer than 8 positions would need copies of less than a swizzle's rows
    if (a.vec && a.v.page_log2 >= 3 && pool_maps<HD>(a.v, &maps))
        return a.R <= 8 ? launch<CaTensor<HD, 1>>(a, maps, sms, kernels, st) : launch<CaTensor<HD, 2>>(a, maps, sms, kernels, st);
    return launch<CaCores<bf16, HD>>(a, {}, sms, kernels, st);
}

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
    ca_common(a, s, v, w, Q, n_q, n_tok, n_sink, window, out, ws);
    a.vec = cache_vec(v, s.dtype == 0 ? 4 : 2);
    if (s.dtype != 0) return s.hd == 64 ? launch_bf16<64>(a, s.sms, kernels, st) : launch_bf16<128>(a, s.sms, kernels, st);
    return s.hd == 64 ? launch<CaCores<float, 64>>(a, {}, s.sms, kernels, st) : launch<CaCores<float, 128>>(a, {}, s.sms, kernels, st);
}

}  // namespace mone

