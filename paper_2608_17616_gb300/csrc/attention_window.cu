// Windowed attention (mone_window_attention): many query rows on the tensor cores (bf16 with 16-byte-aligned rows), and
// the CUDA-core form.  (Few rows on the tensor cores: attention.cu's decode form.)
//
// On the tensor cores, a tile is 128 MMA rows: rt = 128 / group tokens of each of a KV head's `group` query heads, which share
// every staged key and value row.  A CTA takes pairs of tiles of consecutive tokens, which share the staged keys and values too,
// one after another (hd 64: two CTAs an SM, hd 128: one; TMEM holds no more).  Per chunk of 64 keys and tile: S = Q K^T into
// TMEM, the softmax, whose bf16 probabilities go over the scores as the A operand of O += P V, O in TMEM.  A tile has two S
// buffers at hd 128, one at hd 64, where the other three tiles of the SM fill the wait.
// Four warps for each tile do the softmax and the output, a thread a row (= TMEM lane).  (Two threads a row, one tile at a time
// at hd 64 and two at hd 128: 282 us for 223 at 16 layers of 32 heads over 8, 2048 tokens, window 512, hd 64, and 755 for 700 at
// 16001 tokens, window 4096, hd 128.)  Then the loader: keys and values by TMA with the caller's strides through a ring each,
// the queries into a buffer of their own.  Then the MMA issuers, of each tile's S, NB chunks ahead, and of P V.  Loads and S run on
// over the end of a tile (a window has few chunks, so a tile's first loads and last output would otherwise cost as much as
// its chunks): the chunks of all tiles of a CTA are one sequence.
//
// The softmax does without a maximum for each chunk: the scale of a row is the max of its first sixteen keys of which one counts,
// and floating point does not mind later scores above it.  A row whose sum has passed SUM_MOST is scaled down before the next chunk;
// one that overflows within a chunk, by scores some 46 above all before, is computed again at the end, by its warp, like one that met
// a value that is not finite (0.3 to 0.8 ms a row and 4096 positions; a tile that sees such a value has 128 of them).
// At hd 64 the warps' latencies and issue bound it (16 softmax warps an SM: 174 us, 785 TFLOP/s of what the tokens see, at the sizes above,
// 1080 over all of 8000 tokens), at hd 128 the tensor pipe, 70% active (692 us, 1550 TFLOP/s; 740, 1450, at the power cap).
#include <algorithm>
#include <cfloat>
#include <climits>
#include <type_traits>

#include "attention_common.cuh"
#include "per_device.h"

namespace mone {

namespace {

template <int HD>
struct WinSmem {
    static constexpr int CTAS = HD == 64 ? 2 : 1;          // CTAs an SM
    static constexpr int NK = 64;                          // key positions per chunk
    static constexpr int NB = HD == 64 ? 1 : 2;            // S (and P) buffers of a tile: NB NK + HD TMEM columns
    static constexpr int LOAD_WARP = 8, S_WARP = LOAD_WARP + 1, PV_WARP = S_WARP + 2, THREADS = (PV_WARP + 1) * 32;
    static constexpr int TILE_COLS = HD == 64 ? 128 : 256, TMEM = 2 * TILE_COLS;
    static constexpr int QB = HD == 64 ? 2 : 1;            // query buffers, of a pair each
    static constexpr int Q_SLAB = 128 * 128, Q_TILE = (HD / 64) * Q_SLAB;  // 128 query rows x 64 bf16; x HD
    static constexpr int SLAB = NK * 128, TILE = (HD / 64) * SLAB;         // NK keys x 64 bf16; x HD
    static constexpr int NS = HD == 64 ? 2 : 4;            // slots of the ring of keys and of that of values, a chunk each
    static constexpr int K_OFF = QB * 2 * Q_TILE, V_OFF = K_OFF + NS * TILE;
    // qfull[QB] qempty[QB] kfull[NS] kempty[NS] vfull[NS] vempty[NS], and for each tile sfull[NB] odone[NB] pready[NB] oempty
    static constexpr int BAR_OFF = V_OFF + NS * TILE, TILE_BARS = 3 * NB + 1;
    static constexpr int SLOT_OFF = BAR_OFF + (2 * QB + 4 * NS + 2 * TILE_BARS) * 8;
    static constexpr int DYN = SLOT_OFF + 16 + 1024;       // + TMEM slot and count of rows, + alignment slack
    static_assert(NB * NK + HD <= TILE_COLS && CTAS * TMEM <= 512 && CTAS * (DYN + 1024) <= 228 * 1024, "CTAs an SM");
};

// A row's sum is scaled down when it has passed this: far enough above 1 to be rare (with 2^20, scores of standard deviation 4 took
// 904 us for 658 at 16001 tokens, window 4096, hd 128), far enough below FLT_MAX that a chunk seldom gets from there to it
constexpr float SUM_MOST = 0x1p60f;

__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// The same, NaN if one is
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// The two bf16 of p to the two sums of l, in 32 bits
__device__ __forceinline__ void add_bf16x2(uint64_t& l, uint32_t p) {
    asm("{\n\t.reg .b16 lo, hi;\n\t.reg .f32 a, b;\n\t"
        "mov.b32 {lo, hi}, %1;\n\tmov.b64 {a, b}, %0;\n\t"
        "add.f32.bf16 a, lo, a;\n\tadd.f32.bf16 b, hi, b;\n\t"
        "mov.b64 %0, {a, b};\n\t}"
        : "+l"(l)
        : "r"(p));
}

__device__ __forceinline__ float sum_f32x4(const uint64_t (&x)[2]) {
    const float2 s = unpack_f32x2(add_f32x2(x[0], x[1]));
    return s.x + s.y;
}

// The loader and the MMA issuers run their loops as whole warps, so that the compiler keeps descriptors, coordinates and
// addresses in uniform registers, where the instructions want them; the lane with `me` issues.  (With the loop in one lane's
// branch, each of the dozen small MMAs and copies of a chunk came with a handful of moves into them, and these warps, which
// share their schedulers with softmax warps, were the slowest part of the chain.)
__device__ __forceinline__ void win_load_5d(uint32_t dst, const CUtensorMap* m, uint32_t bar, int x, int y, int z, int w, int v, uint32_t me) {
    asm volatile(
        "{\n\t.reg .pred e;\n\t"
        "setp.ne.b32 e, %8, 0;\n\t"
        "@e cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%3, %4, %5, %6, %7}], [%2];\n\t}" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(x), "r"(y), "r"(z), "r"(w), "r"(v), "r"(me)
        : "memory");
}
__device__ __forceinline__ void win_expect(uint32_t bar, uint32_t bytes, uint32_t me) {
    asm volatile(
        "{\n\t.reg .pred e;\n\t"
        "setp.ne.b32 e, %2, 0;\n\t"
        "@e mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n\t}" ::"r"(bar),
        "r"(bytes), "r"(me)
        : "memory");
}
__device__ __forceinline__ void win_mma(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate, uint32_t me) {
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "setp.ne.b32 e, %5, 0;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
        "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(me)
        : "memory");
}
// The same with A in TMEM.
__device__ __forceinline__ void win_mma_ta(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accumulate, uint32_t me) {
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "setp.ne.b32 e, %5, 0;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
        "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(me)
        : "memory");
}
__device__ __forceinline__ void win_commit(uint32_t bar, uint32_t me) {
    asm volatile(
        "{\n\t.reg .pred e;\n\t"
        "setp.ne.b32 e, %1, 0;\n\t"
        "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar),
        "r"(me)
        : "memory");
}

// mbar_wait by a whole warp, with one answer.  It gives up when neither the barrier's phase nor the count of rows computed again has
// moved for the limit: a warp may have 32 such rows between two tiles, each over up to 2^20 positions (0.2 s).
__device__ __forceinline__ bool win_wait(uint32_t bar, uint32_t parity, int* status, const volatile uint32_t* again) {
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
    uint32_t rows = __shfl_sync(0xffffffffu, *again, 0);
    uint64_t t0 = globaltimer_ns();
    while (true) {
#pragma unroll 1
        for (int i = 0; i < 32; ++i)
            if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
        if (__any_sync(0xffffffffu, globaltimer_ns() - t0 > kWaitLimitNs)) {
            const uint32_t now = __shfl_sync(0xffffffffu, *again, 0);
            if (now == rows) {
                atomicOr(status, DEV_TIMEOUT);
                return false;
            }
            rows = now;
            t0 = globaltimer_ns();
        }
    }
}

// row_again by a warp, which has HD / 32 dimensions a lane; eight keys' loads under way
template <int HD>
__device__ __noinline__ void row_by_warp(const bf16* q, const bf16* K, const bf16* V, int vis, const AttnArgs& a, bf16* out) {
    constexpr int D = HD / 32, U = 8;
    const int d0 = D * (threadIdx.x & 31);
    float qf[D], o[D] = {}, m = -INFINITY, l = 0.f;
#pragma unroll
    for (int d = 0; d < D; ++d) qf[d] = __bfloat162float(q[d0 + d]) * a.scale;
    auto keys = [&](int j0, int j1) {
        for (int j = j0; j < j1; j += U) {
            bf16 k[U][D], v[U][D];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int d = 0; d < D; ++d) {
                    const long long at = (long long)min(j + u, j1 - 1) * a.s3 + d0 + d;
                    k[u][d] = K[at];
                    v[u][d] = V[at];
                }
            float z[U], mn = m;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float x = 0.f;
#pragma unroll
                for (int d = 0; d < D; ++d) x = fmaf(qf[d], __bfloat162float(k[u][d]), x);
                z[u] = warp_sum(x);
                if (j + u >= j1) z[u] = -INFINITY;
                mn = fmaxf(mn, z[u]);
            }
            const float corr = m == mn ? 1.f : __expf(m - mn);
            m = mn;
            l *= corr;
#pragma unroll
            for (int d = 0; d < D; ++d) o[d] *= corr;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (z[u] == -INFINITY) continue;
                const float p = __expf(z[u] - mn);
                l += p;
#pragma unroll
                for (int d = 0; d < D; ++d) o[d] = fmaf(p, __bfloat162float(v[u][d]), o[d]);
            }
        }
    };
    const int first = min(a.n_sink, vis);
    keys(0, first);
    keys(max(first, vis - a.window), vis);
    const float inv = l > 0.f ? 1.f / l : l;
#pragma unroll
    for (int d = 0; d < D; ++d) out[d0 + d] = __float2bfloat16_rn(o[d] * inv);
}

// The lowest n bits (n <= 0: none; n >= 32: all)
__device__ __forceinline__ uint32_t low_bits(int n) {
    uint32_t r;
    asm("shl.b32 %0, -1, %1;" : "=r"(r) : "r"(max(n, 0)));  // a shift by 32 or more leaves 0
    return ~r;
}

// The tiles of a CTA, as its warps step through them, pair by pair: the last tokens' come first, of all chains and heads, since
// the first ones see fewer keys, and the CTAs take them in turn, to and fro.  (In the order of the tokens, a CTA's pairs could
// all lie at the same place of their prompts: 223 us for 207 at 16 layers of 32 heads, 2048 tokens, window 512, hd 64.)  What is
// left of the pairs goes by single tiles if there is a CTA for each.
template <int NK>
struct WinTiles {
    int item, step, turn;       // this item, distance to the CTA's next and to the one after that
    int count, whole;           // items in all; those that are pairs
    int np, heads, odd;         // pairs of a KV head; KV heads in all; whether the last pair of a head is one tile
    int c, g, r0, t0, t1;       // chain, KV head, first token; positions of its first and last
    int ns, lo, n, wf, wl;      // chunks of the first positions; first position after them; chunks in all; widths of the last ones
    int wl0;                    // of the last, for the first of two tiles
    bool two;
    __device__ WinTiles(const AttnArgs& a, int C) {
        const int nt = (a.Lq + a.rows - 1) / a.rows, grid = gridDim.x, b = blockIdx.x;
        np = (nt + 1) / 2;
        odd = nt & 1;
        heads = a.n_kv * C;
        const int pairs = np * heads, rest = pairs % grid;
        whole = 2 * rest <= grid ? pairs - rest : pairs;
        count = whole + 2 * (pairs - whole);
        item = b;
        step = 2 * (grid - 1 - b) + 1;
        turn = 2 * b + 1;
    }
    // (the second tile of a head's last pair may not be there; single tiles are a CTA's last)
    __device__ bool more() const { return item < count && !(odd && item >= whole && ((item - whole) & 1) && whole + (item - whole) / 2 < heads); }
    __device__ void next() {
        item += step;
        const int s = step;
        step = turn;
        turn = s;
    }
    __device__ bool has(int x) const { return x == 0 || two; }
    __device__ void open(const AttnArgs& a) {
        const int single = item >= whole, p = single ? whole + (item - whole) / 2 : item, rank = p / heads, cg = p - rank * heads;
        two = !single && !(odd && rank == 0);
        r0 = (2 * (np - 1 - rank) + (single ? (item - whole) & 1 : 0)) * a.rows;
        c = cg / a.n_kv;
        g = cg - c * a.n_kv;
        t0 = a.n_mem + r0;
        t1 = a.n_mem + min(a.Lq, r0 + (two ? 2 : 1) * a.rows) - 1;
        const WinRange w(a, t0, t1, NK);
        ns = w.ns;
        lo = w.lo;
        n = w.n;
        // the last chunk of the first positions may go on into the window
        const int first_end = t0 - a.window + 1 >= ns * NK ? min(a.n_sink, t1 + 1) : t1 + 1;
        wf = (min(NK, first_end - (ns - 1) * NK) + 15) & ~15;
        wl = n > ns ? (min(NK, t1 + 1 - (lo + (n - 1 - ns) * NK)) + 15) & ~15 : wf;
        wl0 = two && n > ns ? max(16, (min(NK, t0 + a.rows - (lo + (n - 1 - ns) * NK)) + 15) & ~15) : wl;
    }
    __device__ int at(int j) const { return j < ns ? j * NK : lo + (j - ns) * NK; }
    // keys of a chunk up to the last that some token of a tile sees, in sixteens: what S, the softmax and P V go over
    __device__ int width(int j, int x) const { return j == n - 1 ? (x ? wl : wl0) : j == ns - 1 ? wf : NK; }
};

template <int HD>
__global__ void __launch_bounds__(WinSmem<HD>::THREADS, WinSmem<HD>::CTAS)
window_prefill_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                      const AttnArgs a, int C) {
    using SM = WinSmem<HD>;
    constexpr int NS = SM::NS, NK = SM::NK, QB = SM::QB, NB = SM::NB;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const uint32_t bars = smem_u32(base + SM::BAR_OFF);
    auto qfull = [&](int i) { return bars + 8 * (i % QB); };  // of the CTA's tile i, phase i / QB
    auto qempty = [&](int i) { return bars + 8 * (QB + i % QB); };
    constexpr int KB0 = 2 * QB, VB0 = KB0 + 2 * NS, SB0 = VB0 + 2 * NS;
    auto kfull = [&](int s) { return bars + 8 * (KB0 + s); };
    auto kempty = [&](int s) { return bars + 8 * (KB0 + NS + s); };
    auto vfull = [&](int s) { return bars + 8 * (VB0 + s); };
    auto vempty = [&](int s) { return bars + 8 * (VB0 + NS + s); };
    // of tile x (of a pair) and chunk j of all the CTA's, phase j / NB
    auto sfull = [&](int x, int j) { return bars + 8 * (SB0 + x * SM::TILE_BARS + j % NB); };
    auto odone = [&](int x, int j) { return bars + 8 * (SB0 + x * SM::TILE_BARS + NB + j % NB); };
    auto pready = [&](int x, int j) { return bars + 8 * (SB0 + x * SM::TILE_BARS + 2 * NB + j % NB); };
    auto oempty = [&](int x) { return bars + 8 * (SB0 + x * SM::TILE_BARS + 3 * NB); };  // of a tile
    uint32_t* slot = reinterpret_cast<uint32_t*>(base + SM::SLOT_OFF);
    uint32_t* again = slot + 1;  // rows computed again
    auto wait = [&](uint32_t bar, uint32_t parity) { return win_wait(bar, parity, a.status, again); };
    // the warp's number from one lane, and below the TMEM address: the compiler then knows them to be the same in all
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    if (tid == 0) {
        *again = 0;
        for (int i = 0; i < QB; ++i) {
            mbar_init(qfull(i), 1);
            mbar_init(qempty(i), 2);
        }
        for (int s = 0; s < NS; ++s) {
            mbar_init(kfull(s), 1);
            mbar_init(kempty(s), 2);
            mbar_init(vfull(s), 1);
            mbar_init(vempty(s), 1);
        }
        for (int x = 0; x < 2; ++x) {
            for (int b = 0; b < NB; ++b) {
                mbar_init(sfull(x, b), 1);
                mbar_init(odone(x, b), 1);
                mbar_init(pready(x, b), 4);
            }
            mbar_init(oempty(x), 4);
        }
        fence_mbar_init();
    }
    if (warp == SM::S_WARP) {
        tmem_alloc(smem_u32(slot), SM::TMEM);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_wait();
    const uint32_t tmem = __shfl_sync(0xffffffffu, *slot, 0);  // of a tile: the S (and P) buffers, then O
    const int rt = a.rows;
    WinTiles<NK> tl(a, C);

    if (warp == SM::LOAD_WARP) {
        const uint32_t me = lane == 0;
        if (me) {
            tma_prefetch_map(&tmQ);
            tma_prefetch_map(&tmK);
            tma_prefetch_map(&tmV);
        }
        bool ok = true;
        // K0 K1 V0 K2 V1 .. over all chunks of all tiles: the keys of a chunk, then the values of the chunk before
        struct Ring {
            int s = 0, ph = 1;  // slot, and the phase of its release (the first round passes)
            __device__ void next() {
                if (++s == NS) {
                    s = 0;
                    ph ^= 1;
                }
            }
        } rk, rv;
        const uint32_t k0 = smem_u32(base + SM::K_OFF), v0 = smem_u32(base + SM::V_OFF);
        int vp = -1, vctx = 0, vlayer = 0, vhead = 0;
        auto load_v = [&]() {
            ok = ok && wait(vempty(rv.s), rv.ph);
            if (!ok) return;
            win_expect(vfull(rv.s), SM::TILE, me);
#pragma unroll
            for (int kb = 0; kb < HD / 64; ++kb)
                win_load_5d(v0 + rv.s * SM::TILE + kb * SM::SLAB, &tmV, vfull(rv.s), 64 * kb, vp, vhead, vlayer, vctx, me);
            rv.next();
        };
        for (int i = 0; ok && tl.more(); ++i, tl.next()) {
            tl.open(a);
            // a dimension that the caches share (stride 0) has one element in the maps
            const int tctx = tl.c / a.L, ctx = a.s0 ? tctx : 0, layer = a.s1 ? tl.c - tctx * a.L : 0, head = a.s2 ? tl.g : 0;
            ok = wait(qempty(i), (i / QB & 1) ^ 1);
            if (!ok) break;
            if (me) {
                mbar_expect_tx(qfull(i), (tl.two ? 2 : 1) * (HD / 64) * a.group * rt * 128);
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int kb = 0; kb < HD / 64 && tl.has(x); ++kb)  // the query rows, [head of the group][token]
                        tma_load_4d(smem_u32(base + (i % QB * 2 + x) * SM::Q_TILE) + kb * SM::Q_SLAB, &tmQ, qfull(i), 64 * kb, tl.r0 + x * rt,
                                    tl.g * a.group, tl.c);
            }
            __syncwarp();
            for (int j = 0; ok && j < tl.n; ++j) {
                const int pos = tl.at(j);
                ok = wait(kempty(rk.s), rk.ph);
                if (!ok) break;
                win_expect(kfull(rk.s), SM::TILE, me);
#pragma unroll
                for (int kb = 0; kb < HD / 64; ++kb)
                    win_load_5d(k0 + rk.s * SM::TILE + kb * SM::SLAB, &tmK, kfull(rk.s), 64 * kb, pos, head, layer, ctx, me);
                rk.next();
                if (vp >= 0) load_v();
                vp = pos;
                vctx = ctx;
                vlayer = layer;
                vhead = head;
            }
        }
        if (vp >= 0) load_v();
        if (!ok) drain_copies();
        __syncwarp();
    } else if (warp >= SM::S_WARP && warp < SM::PV_WARP) {
        // S = Q K^T over HD (K-major both), of one of the tiles
        const uint32_t me = lane == 0, x = warp - SM::S_WARP, t_s = tmem + x * SM::TILE_COLS;
        const uint64_t dq0 = sdesc_sw128(smem_u32(base + x * SM::Q_TILE), 16), dk0 = sdesc_sw128(smem_u32(base + SM::K_OFF), 16);
        bool ok = true;
        int s = 0, ph = 0, J = 0;  // the ring's next slot and its phase; chunk of all the tile's
        for (int i = 0; ok && tl.more(); ++i, tl.next()) {
            tl.open(a);
            ok = wait(qfull(i), i / QB & 1);
            const uint64_t dq = sdesc_step(dq0, i % QB * 2 * SM::Q_TILE);
            for (int j = 0; ok && j < tl.n; ++j) {
                const uint32_t id_s = idesc_bf16_f32(128, tl.width(j, x), false, false);
                const uint64_t dk = sdesc_step(dk0, s * SM::TILE);
                ok = wait(kfull(s), ph);
                if (tl.has(x)) {
                    if (J >= NB) ok = ok && wait(odone(x, J), (J / NB & 1) ^ 1);  // P V of chunk J - NB has read its P, where S goes
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll
                    for (int kb = 0; kb < HD / 64; ++kb)
#pragma unroll
                        for (int u = 0; u < 4; ++u)
                            win_mma(t_s + J % NB * NK, sdesc_step(dq, kb * SM::Q_SLAB + u * 32), sdesc_step(dk, kb * SM::SLAB + u * 32), id_s,
                                    (kb | u) ? 1u : 0u, me);
                    win_commit(sfull(x, J), me);
                    ++J;
                }
                win_commit(kempty(s), me);
                if (++s == NS) {
                    s = 0;
                    ph ^= 1;
                }
            }
            win_commit(qempty(i), me);  // the queries have been read
        }
        if (!ok) drain_copies();
        __syncwarp();
    } else if (warp == SM::PV_WARP) {
        // O += P V over the chunk's keys (P in TMEM, over the scores; V MN-major)
        const uint32_t me = lane == 0, id_o = idesc_bf16_f32(128, HD, false, true);
        const uint64_t dv0 = sdesc_sw128(smem_u32(base + SM::V_OFF), SM::SLAB);
        bool ok = true;
        int s = 0, ph = 0, count[2] = {}, chunk[2] = {};  // ring; items and chunks of each tile
        for (; ok && tl.more(); tl.next()) {
            tl.open(a);
            for (int j = 0; ok && j < tl.n; ++j) {
                const uint64_t dv = sdesc_step(dv0, s * SM::TILE);
                ok = wait(vfull(s), ph);
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    if (!tl.has(x)) continue;
                    const int J = chunk[x]++, wd = tl.width(j, x);
                    const uint32_t t_p = tmem + x * SM::TILE_COLS + J % NB * NK, t_o = tmem + x * SM::TILE_COLS + NB * NK;
                    if (j == 0) ok = ok && wait(oempty(x), (count[x]++ & 1) ^ 1);  // the last tile's O has been read
                    ok = ok && wait(pready(x, J), J / NB & 1);          // P of chunk J is in TMEM
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll
                    for (int kk = 0; kk < NK / 16; ++kk)
                        if (kk * 16 < wd)
                            win_mma_ta(t_o, t_p + kk * 8, sdesc_step(dv, kk * 16 * 128), id_o, (j | kk) ? 1u : 0u, me);
                    win_commit(odone(x, J), me);
                }
                if (!ok) break;
                win_commit(vempty(s), me);
                if (++s == NS) {
                    s = 0;
                    ph ^= 1;
                }
            }
        }
        if (!ok) drain_copies();
        __syncwarp();
    } else {
        // ---- softmax: row = TMEM lane
        const int x = warp >> 2, quarter = warp & 3, row = quarter * 32 + lane, hr = row / rt;
        const float k2 = a.scale * 1.4426950408889634f;  // softmax scale in base 2: exp(s x) = 2^(s log2(e) x)
        const uint32_t t_x = tmem + x * SM::TILE_COLS + ((uint32_t)(quarter * 32) << 16), t_o = t_x + NB * NK;
        bool ok = true;
        int J = 0;  // chunk of all the tile's
        for (; ok && tl.more(); tl.next()) {
            tl.open(a);
            if (!tl.has(x)) continue;
            const int c = tl.c, g = tl.g, r0 = tl.r0 + x * rt;
            const int first = a.n_mem + r0 + 1;                       // keys that the tile's first token sees
            const int keys = a.n_mem + min(a.Lq, r0 + rt);            // its last
            const int tok = tl.r0 + x * rt + row - hr * rt;
            const bool live = hr < a.group && tok < a.Lq;
            const int vis = live ? a.n_mem + tok + 1 : first;         // the row sees keys before it (a row of padding: any)
            // The row's scale; -FLT_MAX: no key counted so far.  A row of padding holds whatever shared memory did (a group that does
            // not divide 128): its sum stays 0 or becomes NaN, and it has no say in the votes below
            float m_run = live ? -FLT_MAX : INFINITY;
            uint64_t l2[2] = {0, 0};
            for (int j = 0; j < tl.n; ++j, ++J) {
                const uint32_t t_s = t_x + J % NB * NK;
                const int at = tl.at(j), wd = tl.width(j, x);
                ok = wait(sfull(x, J), J / NB & 1);
                if (!ok) break;
                tc_fence_after();
                // Hidden keys get scores of -inf, written back: few chunks have any, and the loop over all of them stays short (its
                // instructions, unrolled with masks, did not fit the instruction caches)
                if (at + NK > first || (at + NK > a.n_sink && at < keys - a.window)) {
#pragma unroll 1
                    for (int b = 0; b < NK && b < wd; b += 16) {
                        // sixteen of which some row does not see all (in the window of all: from the last token's first key on)
                        const int p = at + b;
                        if (p + 16 <= first && (p + 16 <= a.n_sink || p >= keys - a.window)) continue;
                        const int nv = vis - p;
                        const uint32_t sees = low_bits(nv) & (~low_bits(nv - a.window) | low_bits(a.n_sink - p));
                        float v[16];
                        uint32_t hid[16];
                        tmem_ld16(t_s + b, v);
#pragma unroll
                        for (int u = 0; u < 16; ++u) hid[u] = sees >> u & 1 ? __float_as_uint(v[u]) : 0xff800000u;
                        tmem_st16(t_s + b, hid);
                    }
                    tmem_wait_st();
                }
                if (__any_sync(0xffffffffu, m_run == -FLT_MAX)) {
                    float cm = -INFINITY;
#pragma unroll 1
                    for (int b = 0; b < NK && b < wd && __any_sync(0xffffffffu, m_run == -FLT_MAX && cm == -INFINITY); b += 16) {
                        float v[16], c16 = -INFINITY;
                        tmem_ld16(t_s + b, v);
#pragma unroll
                        for (int u = 0; u < 16; u += 2) c16 = max3(c16, v[u], v[u + 1]);
                        if (cm == -INFINITY) cm = c16;  // (others may look on: a row's scale is its own)
                    }
                    if (m_run == -FLT_MAX) m_run = fmaxf(cm, -FLT_MAX);  // sums and O are 0 so far
                }
                // (whether or not a row has no scale yet: one whose scores are all NaN never gets one)
                if (__any_sync(0xffffffffu, sum_f32x4(l2) > SUM_MOST)) {
                    const float l = sum_f32x4(l2);
                    ok = wait(odone(x, J - 1), (J - 1) / NB & 1);  // O up to the last chunk
                    if (!ok) break;
                    tc_fence_after();
                    const int e = l > SUM_MOST && l <= FLT_MAX ? ilogbf(l) : 0;  // by a power of two
                    const float corr = ldexpf(1.f, -e);
                    m_run += e / k2;
                    l2[0] = mul_f32x2(l2[0], pack_f32x2(corr, corr));
                    l2[1] = mul_f32x2(l2[1], pack_f32x2(corr, corr));
#pragma unroll 1
                    for (int cb = 0; cb < HD; cb += 16) {
                        float ov[16];
                        uint32_t on[16];
                        tmem_ld16(t_o + cb, ov);
#pragma unroll
                        for (int u = 0; u < 16; ++u) on[u] = __float_as_uint(ov[u] * corr);
                        tmem_st16(t_o + cb, on);
                    }
                }
                const float moff = -m_run * k2;
                const uint64_t kk2 = pack_f32x2(k2, k2), mm2 = pack_f32x2(moff, moff);
                auto probs = [&](auto& v, int b, int n) {
#pragma unroll
                    for (int h = 0; h < n; h += 16) {
                        uint32_t pk[8];
#pragma unroll
                        for (int u = 0; u < 8; ++u) {
                            const float2 z = unpack_f32x2(fma_f32x2(pack_f32x2(v[h + 2 * u], v[h + 2 * u + 1]), kk2, mm2));
                            const float e0 = at_exp2(z.x), e1 = at_exp2(z.y);
                            pk[u] = pack_bf16(e0, e1);
                            // The sums take the probabilities that the MMA sees, so that a row's weights add up to 1.  (Sums of
                            // e0 and e1: error 2.3e-3 of the output for 2.1e-3, the mean of equal values is not that value; 182 us
                            // for 172 at 16 layers of 2048 tokens, hd 64, and 710 for 740 at 16001, hd 128.)
                            add_bf16x2(l2[u & 1], pk[u]);
                        }
                        tmem_st8(t_s + (b + h) / 2, pk);
                    }
                };
                if (wd == NK) {
#pragma unroll
                    for (int b = 0; b < NK; b += 32) {
                        float v[32];
                        tmem_ld32(t_s + b, v);
                        probs(v, b, 32);
                    }
                } else {
#pragma unroll 1
                    for (int b = 0; b < wd; b += 16) {
                        float v[16];
                        tmem_ld16(t_s + b, v);
                        probs(v, b, 16);
                    }
                }
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(pready(x, J));
            }
            if (!ok) break;
            const float sum = sum_f32x4(l2);
            ok = wait(odone(x, J - 1), (J - 1) / NB & 1);
            if (!ok) break;
            tc_fence_after();
            // no key that counts: 0; a sum that has overflowed: NaN, and the row again
            const float inv = sum == 0.f ? 0.f : sum <= FLT_MAX ? 1.f / sum : NAN;
            const size_t at = (((size_t)c * a.n_q + g * a.group + (live ? hr : 0)) * a.Lq + (live ? tok : 0)) * HD;
            bf16* orow = static_cast<bf16*>(a.out) + at;
            float top = 0.f;  // of the row's magnitudes, NaN if one is
#pragma unroll
            for (int cb = 0; cb < HD; cb += 32) {
                float v[32];
                tmem_ld32(t_o + cb, v);
#pragma unroll
                for (int u = 0; u < 32; u += 2) {
                    v[u] *= inv;
                    v[u + 1] *= inv;
                    top = max3_nan(top, fabsf(v[u]), fabsf(v[u + 1]));
                }
                if (live) {
#pragma unroll
                    for (int u = 0; u < 32; u += 8)
                        *reinterpret_cast<uint4*>(orow + cb + u) = make_uint4(pack_bf16(v[u], v[u + 1]), pack_bf16(v[u + 2], v[u + 3]),
                                                                              pack_bf16(v[u + 4], v[u + 5]), pack_bf16(v[u + 6], v[u + 7]));
                }
                __syncwarp();
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(oempty(x));
            const long long kv_off = (long long)(c / a.L) * a.s0 + (long long)(c % a.L) * a.s1 + (long long)g * a.s2;
            for (uint32_t bad = __ballot_sync(0xffffffffu, live && !(top <= FLT_MAX)); bad; bad &= bad - 1) {
                const int src = __ffs(bad) - 1;
                const size_t of = __shfl_sync(0xffffffffu, at, src);
                row_by_warp<HD>(static_cast<const bf16*>(a.Q) + of, static_cast<const bf16*>(a.K) + kv_off, static_cast<const bf16*>(a.V) + kv_off,
                                __shfl_sync(0xffffffffu, vis, src), a, static_cast<bf16*>(a.out) + of);
                if (lane == 0) atomicAdd(again, 1u);
            }
            __syncwarp();
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == SM::S_WARP) tmem_dealloc(tmem, SM::TMEM);
}

// ---------------------------------------------------------------- CUDA cores: fp32, and bf16 rows that are not aligned
// 32 rows (query heads x tokens of a KV head) a CTA, chunks of 64 keys as fp32 in shared memory.  Both products are tiled in
// registers, two values an instruction: a thread has 4 rows x 4 keys of S (keys 16 apart), in sums of the even dimensions and of
// the odd, then 4 rows x 4 dimensions (twice at hd 128) of O, eight 16-byte loads for 64 multiply-adds each.  A row's 64 scores
// lie in 16 lanes, which take its max by shuffles; each thread adds up the probabilities that it made itself, and the
// sums meet at the end.  The next chunk's keys are under way during the softmax and P V, its values during the scores.
// Bound by the warps' issue and the loads from shared memory: 2 layers of 8 heads over 4, 700 tokens, window 200, hd 64 take
// 27 us (35 without the copies ahead, one multiply-add an instruction and the first tokens first); 4 layers of 32 over 8,
// 2000 tokens, window 512 829 us (964), 37 TFLOP/s.
constexpr int WC_R = 4, WC_ROWS = 32, WC_KEYS = 64, WC_THREADS = 16 * WC_ROWS / WC_R;  // WC_R: rows of a thread

template <int HD>
struct WcSmem {
    static constexpr int P = HD + 4;          // floats between rows: 16 lanes' 16-byte loads of a column fall on different banks
    static constexpr int PP = WC_KEYS + 4;
    static constexpr int K = WC_ROWS * P, V = K + WC_KEYS * P, PR = V + WC_KEYS * P, FLOATS = PR + WC_ROWS * PP;
};

// Row i of `n` (n: the rows that are there) of HD elements from `row(i)`, as fp32 times `scale`; zeros after the last.
template <typename T, int HD, int ROWS, typename Row>
__device__ __forceinline__ void wc_stage(float* dst, int n, bool vec, float scale, Row&& row) {
    constexpr int PER = 16 / sizeof(T), VPR = HD / PER;
    if (vec) {
#pragma unroll 8
        for (int e = threadIdx.x; e < ROWS * VPR; e += WC_THREADS) {
            const int i = e / VPR, u = e % VPR;
            // (fp32: after the wait for the kernel ahead)
            const uint4* p = i < n ? reinterpret_cast<const uint4*>(row(i)) + u : nullptr;
            const uint4 r = !p ? make_uint4(0, 0, 0, 0) : sizeof(T) == 4 ? *p : __ldg(p);
            const T* t = reinterpret_cast<const T*>(&r);
#pragma unroll
            for (int k = 0; k < PER; k += 4)
                *reinterpret_cast<float4*>(dst + i * WcSmem<HD>::P + u * PER + k) =
                    make_float4(to_f<T>(t[k]) * scale, to_f<T>(t[k + 1]) * scale, to_f<T>(t[k + 2]) * scale, to_f<T>(t[k + 3]) * scale);
        }
    } else {
        for (int e = threadIdx.x; e < ROWS * HD; e += WC_THREADS) {
            const int i = e / HD, d = e % HD;
            dst[i * WcSmem<HD>::P + d] = i < n ? to_f<T>(row(i)[d]) * scale : 0.f;
        }
    }
}

__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// The same, unscaled, of which fp32 rows may still be under way
template <typename T, int HD, int ROWS, typename Row>
__device__ __forceinline__ void wc_copy(float* dst, int n, bool vec, Row&& row) {
    if (sizeof(T) != 4 || !vec) return wc_stage<T, HD, ROWS>(dst, n, vec, 1.f, row);
    constexpr int VPR = HD / 4;
#pragma unroll 4
    for (int e = threadIdx.x; e < ROWS * VPR; e += WC_THREADS) {
        const int i = e / VPR, u = e % VPR;
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst + i * WcSmem<HD>::P + 4 * u)),
                     "l"(row(i < n ? i : 0) + 4 * u), "r"(i < n ? 16 : 0)  // zeros after the last
                     : "memory");
    }
}

template <typename T, int HD>
__global__ void __launch_bounds__(WC_THREADS) window_cores_kernel(const AttnArgs a, int hb, int head_blocks, int C, bool vec_q) {
    using SM = WcSmem<HD>;
    constexpr int DB = HD / 64;  // blocks of 64 dimensions
    extern __shared__ float sh[];
    float *Qs = sh, *Ks = sh + SM::K, *Vs = sh + SM::V, *Ps = sh + SM::PR;
    // the last tokens first, of all chains and heads: the first ones, which see fewer keys, fill the gaps at the end
    const int heads_all = C * a.n_kv * head_blocks, rank = blockIdx.x / heads_all, cgh = blockIdx.x - rank * heads_all;
    const int cg = cgh / head_blocks, h0 = (cgh - cg * head_blocks) * hb, c = cg / a.n_kv, g = cg - c * a.n_kv;
    const int r0 = ((a.Lq + a.rows - 1) / a.rows - 1 - rank) * a.rows, heads = min(hb, a.group - h0), toks = min(a.rows, a.Lq - r0), rows = heads * toks;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const long long kv_off = (long long)(c / a.L) * a.s0 + (long long)(c % a.L) * a.s1 + (long long)g * a.s2;
    const T* Kc = static_cast<const T*>(a.K) + kv_off;
    const T* Vc = static_cast<const T*>(a.V) + kv_off;
    if constexpr (sizeof(T) == 4) pdl_wait();
    // row i of the tile: head h0 + i / toks, token r0 + i % toks
    auto q_at = [&](int i) { return (((size_t)c * a.n_q + (size_t)g * a.group + h0 + i / toks) * a.Lq + r0 + i % toks) * HD; };
    wc_stage<T, HD, WC_ROWS>(Qs, rows, vec_q, a.scale, [&](int i) { return static_cast<const T*>(a.Q) + q_at(i); });
    float m[WC_R], l[WC_R];
    uint64_t o[WC_R][2 * DB];
    int vis[WC_R];
#pragma unroll
    for (int i = 0; i < WC_R; ++i) {
        const int row = WC_R * ty + i;
        vis[i] = row < rows ? a.n_mem + r0 + row % toks + 1 : 0;
        m[i] = -INFINITY;
        l[i] = 0.f;
#pragma unroll
        for (int d = 0; d < 2 * DB; ++d) o[i][d] = 0;
    }
    const int keys = a.n_mem + r0 + toks;
    const WinRange win(a, a.n_mem + r0, keys - 1, WC_KEYS);
    // keys of a chunk up to the last that some row sees
    auto there = [&](int ch) {
        const bool first_only = ch < win.ns && a.n_mem + r0 - a.window + 1 >= (ch + 1) * WC_KEYS;
        return min(WC_KEYS, (first_only ? min(a.n_sink, keys) : keys) - win.at(ch, WC_KEYS));
    };
    auto stage = [&](float* dst, const T* src, int ch) {
        if (ch >= win.n) return;
        const int j0 = win.at(ch, WC_KEYS);
        wc_copy<T, HD, WC_KEYS>(dst, there(ch), a.vec, [&](int i) { return src + (long long)(j0 + i) * a.s3; });
    };
    // a chunk's keys are under way from the last one's scores on, its values from the last one's products
    stage(Ks, Kc, 0);
    cp_async_commit();
    stage(Vs, Vc, 0);
    cp_async_commit();
    for (int ch = 0; ch < win.n; ++ch) {
        const int j0 = win.at(ch, WC_KEYS), nk = there(ch), nj = (nk + 15) / 16;  // and the sixteens of them
        cp_async_wait<1>();
        __syncthreads();
        float s[WC_R][4];
        uint64_t s2[WC_R][4];  // of the even dimensions and of the odd
#pragma unroll
        for (int i = 0; i < WC_R; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) s2[i][j] = 0;
        auto scores = [&](auto all) {  // all: of the four sixteens
#pragma unroll 4
            for (int d = 0; d < HD; d += 4) {
                ulonglong2 q[WC_R];
#pragma unroll
                for (int i = 0; i < WC_R; ++i) q[i] = *reinterpret_cast<const ulonglong2*>(Qs + (WC_R * ty + i) * SM::P + d);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (!decltype(all)::value && j >= nj) break;
                    const ulonglong2 k = *reinterpret_cast<const ulonglong2*>(Ks + (tx + 16 * j) * SM::P + d);
#pragma unroll
                    for (int i = 0; i < WC_R; ++i) s2[i][j] = fma_f32x2(q[i].x, k.x, fma_f32x2(q[i].y, k.y, s2[i][j]));
                }
            }
        };
        if (nj == 4)
            scores(std::true_type());
        else
            scores(std::false_type());
        __syncthreads();
        stage(Ks, Kc, ch + 1);
        cp_async_commit();
#pragma unroll
        for (int i = 0; i < WC_R; ++i) {
            float mn = m[i];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 x = unpack_f32x2(s2[i][j]);
                s[i][j] = x.x + x.y;
                const int p = j0 + tx + 16 * j;
                s[i][j] = p < j0 + nk && p < vis[i] && (p < a.n_sink || p >= vis[i] - a.window) ? s[i][j] : -INFINITY;
                mn = fmaxf(mn, s[i][j]);
            }
#pragma unroll
            for (int x = 1; x < 16; x <<= 1) mn = fmaxf(mn, __shfl_xor_sync(0xffffffffu, mn, x));
            const float corr = mn == m[i] ? 1.f : __expf(m[i] - mn), off = mn == -INFINITY ? 0.f : mn;
            m[i] = mn;
            l[i] *= corr;
#pragma unroll
            for (int d = 0; d < 2 * DB; ++d) o[i][d] = mul_f32x2(o[i][d], pack_f32x2(corr, corr));
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float p = __expf(s[i][j] - off);
                l[i] += p;
                Ps[(WC_R * ty + i) * SM::PP + tx + 16 * j] = p;
            }
        }
        cp_async_wait<1>();
        __syncthreads();  // (a row's probabilities are its own half-warp's)
#pragma unroll 4
        for (int k = 0; k < nk; k += 4) {  // to a multiple of 4: zeros
            float4 p[WC_R];
#pragma unroll
            for (int i = 0; i < WC_R; ++i) p[i] = *reinterpret_cast<const float4*>(Ps + (WC_R * ty + i) * SM::PP + k);
#pragma unroll
            for (int b = 0; b < DB; ++b) {
                ulonglong2 v[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) v[u] = *reinterpret_cast<const ulonglong2*>(Vs + (k + u) * SM::P + 64 * b + 4 * tx);
#pragma unroll
                for (int i = 0; i < WC_R; ++i) {
                    const float pi[4] = {p[i].x, p[i].y, p[i].z, p[i].w};
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const uint64_t pp = pack_f32x2(pi[u], pi[u]);
                        o[i][2 * b] = fma_f32x2(pp, v[u].x, o[i][2 * b]);
                        o[i][2 * b + 1] = fma_f32x2(pp, v[u].y, o[i][2 * b + 1]);
                    }
                }
            }
        }
        __syncthreads();
        stage(Vs, Vc, ch + 1);
        cp_async_commit();
    }
#pragma unroll
    for (int i = 0; i < WC_R; ++i) {
        const int row = WC_R * ty + i;
#pragma unroll
        for (int x = 1; x < 16; x <<= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], x);
        if (row >= rows) continue;
        const float inv = l[i] == 0.f ? 0.f : 1.f / l[i];  // no key that counts: 0
        const size_t at = q_at(row);
#pragma unroll
        for (int b = 0; b < DB; ++b) {
            T* out = static_cast<T*>(a.out) + at + 64 * b + 4 * tx;
            const float2 x = unpack_f32x2(o[i][2 * b]), y = unpack_f32x2(o[i][2 * b + 1]);
            float w[4] = {x.x * inv, x.y * inv, y.x * inv, y.y * inv};
            bool bad = false;
#pragma unroll
            for (int d = 0; d < 4; ++d) bad |= !isfinite(w[d]);
            if (bad) row_again<T, HD, 4, 1>(static_cast<const T*>(a.Q) + at, Kc, Vc, a.s3, vis[i], a, 64 * b + 4 * tx, w);
            for (int d = 0; d < 4; ++d) out[d] = from_f<T>(w[d]);
        }
    }
}

template <typename T, int HD>
cudaError_t launch_cores(AttnArgs a, int C, cudaStream_t st) {
    constexpr size_t smem = WcSmem<HD>::FLOATS * sizeof(float);
    static PerDevice<SmemOptIn> once;
    cudaError_t e = smem_opt_in(reinterpret_cast<const void*>(window_cores_kernel<T, HD>), smem, once);
    if (e != cudaSuccess) return e;
    const int hb = std::min(a.group, WC_ROWS), head_blocks = (a.group + hb - 1) / hb;
    a.rows = WC_ROWS / hb;  // tokens of a tile
    const long long blocks = (long long)((a.Lq + a.rows - 1) / a.rows) * head_blocks * a.n_kv * C;
    if (blocks > INT_MAX) return cudaErrorInvalidConfiguration;
    // (programmatic: fp32, whose keys and values come by asynchronous copies)
    return launch_kernel(window_cores_kernel<T, HD>, dim3((unsigned)blocks), dim3(WC_THREADS), smem, st, sizeof(T) == 4, 1, a, hb, head_blocks, C,
                         (reinterpret_cast<uintptr_t>(a.Q) & 15u) == 0);
}

template <int HD>
cudaError_t launch(AttnArgs a, int n_ctx, int C, int sms, cudaStream_t st) {
    static PerDevice<SmemOptIn> once;
    cudaError_t e = smem_opt_in(reinterpret_cast<const void*>(window_prefill_kernel<HD>), WinSmem<HD>::DYN, once);
    if (e != cudaSuccess) return e;
    // The maps of the last call's shape, of which a call only sets the addresses
    struct Plan {
        long long key[10];
        CUtensorMap q, kv;
    };
    static thread_local Plan plan = {};
    const int rows = 128 / a.group;  // tokens per tile: the group's heads x rows fill the 128 MMA rows
    const long long key[10] = {n_ctx, a.L, a.n_q, a.n_kv, a.Lq, a.n_mem, a.s0, a.s1, a.s2, a.s3};
    if (!std::equal(key, key + 10, plan.key)) {
        const uint64_t Lq = a.Lq, keys = (uint64_t)a.n_mem + Lq;
        const uint64_t qd[4] = {HD, Lq, (uint64_t)a.n_q, (uint64_t)C}, qs[3] = {HD * 2, Lq * HD * 2, a.n_q * Lq * HD * 2};
        const uint32_t qb[4] = {64, (uint32_t)rows, (uint32_t)a.group, 1};
        // the caller's strides; a dimension that the caches share (stride 0) has one element, which takes any stride
        const uint64_t kd[5] = {HD, keys, a.s2 ? (uint64_t)a.n_kv : 1, a.s1 ? (uint64_t)a.L : 1, a.s0 ? (uint64_t)n_ctx : 1};
        const uint64_t s3 = a.s3 * 2;
        const uint64_t ks[4] = {s3, kd[2] > 1 ? a.s2 * 2 : s3, kd[3] > 1 ? a.s1 * 2 : s3, kd[4] > 1 ? a.s0 * 2 : s3};
        const uint32_t kb[5] = {64, WinSmem<HD>::NK, 1, 1, 1};
        plan.key[0] = 0;
        if (!encode_map_bf16_4d(&plan.q, a.Q, qd, qs, qb) || !encode_map_bf16_5d(&plan.kv, a.K, kd, ks, kb)) return cudaErrorNotSupported;
        std::copy(key, key + 10, plan.key);
    }
    CUtensorMap mq = plan.q, mk = plan.kv, mv = plan.kv;
    if (!retarget_map(&mq, a.Q) || !retarget_map(&mk, a.K) || !retarget_map(&mv, a.V)) return cudaErrorInvalidValue;
    a.rows = rows;
    const long long nt = (a.Lq + rows - 1) / rows, pairs = (nt + 1) / 2 * a.n_kv * C, ctas = (long long)WinSmem<HD>::CTAS * sms;
    if (pairs >= 1ll << 29) return cudaErrorNotSupported;
    const long long grid = 2 * pairs <= ctas ? 2 * pairs : std::min(pairs, ctas);  // single tiles if there is a CTA for each
    return launch_kernel(window_prefill_kernel<HD>, dim3((unsigned)grid), dim3(WinSmem<HD>::THREADS), WinSmem<HD>::DYN, st, true, 1, mq, mk, mv, a, C);
}

}  // namespace

cudaError_t launch_window_cores(AttnArgs a, int dtype, int hd, int C, cudaStream_t st) {
    if (dtype == 0) return hd == 64 ? launch_cores<float, 64>(a, C, st) : launch_cores<float, 128>(a, C, st);
    return hd == 64 ? launch_cores<bf16, 64>(a, C, st) : launch_cores<bf16, 128>(a, C, st);
}

cudaError_t launch_window_prefill(const AttnArgs& a, int hd, int n_ctx, int C, int sms, cudaStream_t st) {
    return hd == 64 ? launch<64>(a, n_ctx, C, sms, st) : launch<128>(a, n_ctx, C, sms, st);
}

}  // namespace mone
