// Windowed attention of many query rows (mone_window_attention, bf16 with 16-byte-aligned rows) on the tensor cores.
//
// A tile is 128 MMA rows: rt = 128 / group tokens of each of a KV head's `group` query heads, which share every staged key
// and value row.  A CTA, two an SM, takes one tile after another.  Per chunk of NK keys: S = Q K^T into one of two TMEM
// buffers, the softmax by one thread a row, whose bf16 probabilities go over the scores as the A operand of O += P V, O in TMEM.
// Warps 0-3: the softmax, row = thread = TMEM lane, and the output.  Warp 4: the loader; keys and values by TMA with the caller's
// strides through a ring of NS slots, the queries into a buffer of their own.  Warp 5: the MMA issuer, two chunks of S ahead of
// P V.  Loads and S run on over the end of a tile (a window has few chunks, so a tile's first loads and last output would
// otherwise cost as much as its chunks): the chunks of all tiles of a CTA are one sequence.
#include <algorithm>
#include <cfloat>

#include "attention_common.cuh"
#include "per_device.h"

namespace mone {

namespace {

template <int HD>
struct WinSmem {
    static constexpr int LOAD_WARP = 4, MMA_WARP = 5, THREADS = 6 * 32;
    static constexpr int NK = HD == 64 ? 96 : 64;          // key positions per chunk: 2 NK + HD TMEM columns
    static constexpr int TMEM = 256;                       // two CTAs an SM
    static constexpr int QB = HD == 64 ? 2 : 1;            // query buffers
    static constexpr int Q_SLAB = 128 * 128, Q_TILE = (HD / 64) * Q_SLAB;  // 128 query rows x 64 bf16; x HD
    static constexpr int SLAB = NK * 128, TILE = (HD / 64) * SLAB;         // NK keys x 64 bf16; x HD
    static constexpr int NS = HD == 64 ? 6 : 4;            // ring slots, one K or V chunk each
    static constexpr int KV_OFF = QB * Q_TILE;
    static constexpr int BAR_OFF = KV_OFF + NS * TILE;     // qfull[QB] qempty[QB] full[NS] empty[NS] sfull[2] odone[2] pready[2] oempty
    static constexpr int SLOT_OFF = BAR_OFF + (2 * QB + 2 * NS + 7) * 8;
    static constexpr int DYN = SLOT_OFF + 16 + 1024;       // + TMEM slot, + alignment slack
};
static_assert(2 * (WinSmem<64>::DYN + 1024) <= 228 * 1024 && 2 * (WinSmem<128>::DYN + 1024) <= 228 * 1024, "two CTAs an SM");

__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// The tiles of a CTA and their chunks, as its warps step through them
struct WinTiles {
    int tile, step, count, nt;  // this tile, distance to the CTA's next, tiles in all, of a KV head
    __device__ WinTiles(const AttnArgs& a, int C) {
        nt = (a.Lq + a.rows - 1) / a.rows;
        tile = blockIdx.x;
        step = gridDim.x;
        count = nt * a.n_kv * C;
    }
    __device__ bool more() const { return tile < count; }
    __device__ void next() { tile += step; }
    __device__ void where(const AttnArgs& a, int& c, int& g, int& r0) const {
        const int cg = tile / nt;
        r0 = (tile - cg * nt) * a.rows;
        c = cg / a.n_kv;
        g = cg - c * a.n_kv;
    }
};

template <int HD>
__global__ void __launch_bounds__(WinSmem<HD>::THREADS, 2)
window_prefill_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                      const AttnArgs a, int C) {
    using SM = WinSmem<HD>;
    constexpr int NS = SM::NS, NK = SM::NK, QB = SM::QB;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const uint32_t bars = smem_u32(base + SM::BAR_OFF);
    auto qfull = [&](int i) { return bars + 8 * (i % QB); };  // of the CTA's tile i, phase i / QB
    auto qempty = [&](int i) { return bars + 8 * (QB + i % QB); };
    auto full = [&](int s) { return bars + 8 * (2 * QB + s); };
    auto empty = [&](int s) { return bars + 8 * (2 * QB + NS + s); };
    // of chunk j of all the CTA's, phase j >> 1
    auto sfull = [&](int j) { return bars + 8 * (2 * QB + 2 * NS + (j & 1)); };
    auto odone = [&](int j) { return bars + 8 * (2 * QB + 2 * NS + 2 + (j & 1)); };
    auto pready = [&](int j) { return bars + 8 * (2 * QB + 2 * NS + 4 + (j & 1)); };
    const uint32_t oempty = bars + 8 * (2 * QB + 2 * NS + 6);  // of a tile
    uint32_t* slot = reinterpret_cast<uint32_t*>(base + SM::SLOT_OFF);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int i = 0; i < QB; ++i) {
            mbar_init(qfull(i), 1);
            mbar_init(qempty(i), 1);
        }
        for (int s = 0; s < NS; ++s) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(sfull(b), 1);
            mbar_init(odone(b), 1);
            mbar_init(pready(b), 4);  // the softmax warps
        }
        mbar_init(oempty, 4);
        fence_mbar_init();
    }
    if (warp == SM::MMA_WARP) {
        tmem_alloc(smem_u32(slot), SM::TMEM);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *slot, t_out = tmem + 2 * NK;  // two S (and P) buffers, then O
    const int rt = a.rows;
    WinTiles tl(a, C);
    // a tile's chunks: of the keys that its tokens r0 .. see
    auto range = [&](int r0) { return WinRange(a, a.n_mem + r0, a.n_mem + min(a.Lq, r0 + rt) - 1, NK); };

    if (warp == SM::LOAD_WARP) {
        if (lane == 0) {
            tma_prefetch_map(&tmQ);
            tma_prefetch_map(&tmK);
            tma_prefetch_map(&tmV);
            int s = 0, ph = 1;  // slot, and the phase of its release (the first round passes)
            bool ok = true;
            auto load = [&](const CUtensorMap* m, int pos, int c, int g) {
                ok = ok && mbar_wait(empty(s), ph, a.status);
                if (!ok) return;
                const uint32_t dst = smem_u32(base + SM::KV_OFF + s * SM::TILE);
                // a dimension that the caches share (stride 0) has one element in the maps
                const int ctx = a.s0 ? c / a.L : 0, layer = a.s1 ? c % a.L : 0, head = a.s2 ? g : 0;
                mbar_expect_tx(full(s), SM::TILE);
#pragma unroll
                for (int kb = 0; kb < HD / 64; ++kb)
                    tma_load_5d(dst + kb * SM::SLAB, m, full(s), 64 * kb, pos, head, layer, ctx);
                if (++s == NS) {
                    s = 0;
                    ph ^= 1;
                }
            };
            // K0 K1 V0 K2 V1 .. over all chunks of all tiles: the keys of a chunk, then the values of the chunk before
            int vp = -1, vc = 0, vg = 0;
            for (int i = 0; ok && tl.more(); ++i, tl.next()) {
                int c, g, r0;
                tl.where(a, c, g, r0);
                const WinRange w = range(r0);
                ok = mbar_wait(qempty(i), (i / QB & 1) ^ 1, a.status);
                if (!ok) break;
                mbar_expect_tx(qfull(i), (HD / 64) * a.group * rt * 128);
#pragma unroll
                for (int kb = 0; kb < HD / 64; ++kb)  // the query rows, [head of the group][token]
                    tma_load_4d(smem_u32(base + (i % QB) * SM::Q_TILE) + kb * SM::Q_SLAB, &tmQ, qfull(i), 64 * kb, r0, g * a.group, c);
                for (int j = 0; ok && j < w.n; ++j) {
                    load(&tmK, w.at(j, NK), c, g);
                    if (vp >= 0) load(&tmV, vp, vc, vg);
                    vp = w.at(j, NK);
                    vc = c;
                    vg = g;
                }
            }
            if (vp >= 0) load(&tmV, vp, vc, vg);
            if (!ok) drain_copies();
        }
        __syncwarp();
    } else if (warp == SM::MMA_WARP) {
        if (lane == 0) {
            const uint32_t id_s = idesc_bf16_f32(128, NK, false, false), id_o = idesc_bf16_f32(128, HD, false, true);
            // descriptors of the queries and of the ring's first slot as K and as V
            const uint64_t dq0 = sdesc_sw128(smem_u32(base), 16), dk0 = sdesc_sw128(smem_u32(base + SM::KV_OFF), 16),
                           dv0 = sdesc_sw128(smem_u32(base + SM::KV_OFF), SM::SLAB);
            int s = 0, ph = 0;  // the ring's next slot and its phase
            bool ok = true;
            auto next = [&]() {
                if (++s == NS) {
                    s = 0;
                    ph ^= 1;
                }
            };
            // S runs two chunks ahead of P V, on into the CTA's next tile
            int si = 0, sj = 0, sn = 0, SJ = 0;  // S: tile, chunk in it, its chunks, chunk of all
            auto open = [&]() {
                int c, g, r0;
                tl.where(a, c, g, r0);
                sn = range(r0).n;
                sj = 0;
            };
            auto issue_s = [&]() {  // S = Q K^T over HD (K-major both)
                if (!ok || !tl.more()) return;
                if (sj == 0) {
                    open();
                    ok = mbar_wait(qfull(si), si / QB & 1, a.status);
                }
                ok = ok && mbar_wait(full(s), ph, a.status);
                if (!ok) return;
                tc_fence_after();
                const uint64_t dk = sdesc_step(dk0, s * SM::TILE), dq = sdesc_step(dq0, si % QB * SM::Q_TILE);
#pragma unroll
                for (int kb = 0; kb < HD / 64; ++kb)
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        umma_bf16(tmem + (SJ & 1) * NK, sdesc_step(dq, kb * SM::Q_SLAB + u * 32), sdesc_step(dk, kb * SM::SLAB + u * 32), id_s,
                                  (kb | u) ? 1u : 0u);
                umma_commit(sfull(SJ));
                umma_commit(empty(s));
                next();
                ++SJ;
                if (++sj == sn) {
                    umma_commit(qempty(si));  // the queries have been read
                    ++si;
                    sj = 0;
                    tl.next();
                }
            };
            issue_s();
            issue_s();
            WinTiles pt(a, C);
            int J = 0;
            for (int i = 0; ok && pt.more(); ++i, pt.next()) {
                int c, g, r0;
                pt.where(a, c, g, r0);
                const int n = range(r0).n;
                for (int j = 0; ok && j < n; ++j, ++J) {
                    ok = mbar_wait(full(s), ph, a.status) && mbar_wait(pready(J), (J >> 1) & 1, a.status);  // P of chunk J is in TMEM
                    if (j == 0) ok = ok && mbar_wait(oempty, (i & 1) ^ 1, a.status);  // the last tile's O has been read
                    if (!ok) break;
                    tc_fence_after();
                    const uint64_t dv = sdesc_step(dv0, s * SM::TILE);
#pragma unroll
                    for (int kk = 0; kk < NK / 16; ++kk)  // O += P V over the chunk's keys (P in TMEM, V MN-major)
                        umma_bf16_ta(t_out, tmem + (J & 1) * NK + kk * 8, sdesc_step(dv, kk * 16 * 128), id_o, (j | kk) ? 1u : 0u);
                    umma_commit(odone(J));
                    umma_commit(empty(s));
                    next();
                    // the next S goes over the P that P V has to have read
                    if (tl.more()) {
                        ok = mbar_wait(odone(J), (J >> 1) & 1, a.status);
                        issue_s();
                    }
                }
            }
            if (!ok) drain_copies();
        }
        __syncwarp();
    } else {
        // ---- softmax: row = thread = TMEM lane
        const int row = tid, hr = row / rt;
        const float k2 = a.scale * 1.4426950408889634f;  // softmax scale in base 2: exp(s x) = 2^(s log2(e) x)
        const float grow = 8.f / k2;
        const uint32_t lane_off = (uint32_t)(warp * 32) << 16, t_o = t_out + lane_off;
        bool ok = true;
        int J = 0;
        for (int i = 0; ok && tl.more(); ++i, tl.next()) {
            int c, g, r0;
            tl.where(a, c, g, r0);
            const WinRange win = range(r0);
            const int keys = a.n_mem + min(a.Lq, r0 + rt);  // keys the tile's last token sees
            const int tok = r0 + row - hr * rt;
            const bool live = hr < a.group && tok < a.Lq;
            const int vis = a.n_mem + (live ? tok : r0) + 1;  // the row sees keys before it (a row of padding: any)
            float m_run = 0.f;
            uint64_t l2[2] = {0, 0};
            for (int j = 0; j < win.n; ++j, ++J) {
                const uint32_t t_s = tmem + lane_off + (J & 1) * NK;
                ok = __all_sync(0xffffffffu, mbar_wait(sfull(J), (J >> 1) & 1, a.status));
                if (!ok) break;
                tc_fence_after();
                float v[NK];
                if constexpr (NK == 96)
                    tmem_ld96(t_s, v);
                else
                    tmem_ld64(t_s, v);
                const int p0 = win.at(j, NK);
                // some row does not see the whole chunk (in the window of all: from the last token's first key on)
                if (p0 + NK > a.n_mem + r0 + 1 || (p0 + NK > a.n_sink && p0 < keys - a.window)) {
                    const int nv = vis - p0, nw = vis - a.window - p0, ns = a.n_sink - p0;
#pragma unroll
                    for (int u = 0; u < NK; ++u) v[u] = u < nv && (u >= nw || u < ns) ? v[u] : -INFINITY;
                }
                float c4[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
                for (int u = 4; u < NK; u += 8)
#pragma unroll
                    for (int k = 0; k < 4; ++k) c4[k] = u + 4 < NK ? max3(c4[k], v[u + k], v[u + 4 + k]) : fmaxf(c4[k], v[u + k]);
                const float cm = max3(fmaxf(c4[0], c4[1]), c4[2], c4[3]);
                // The scale is the max of the first chunk, and of a later one where that is over 2^8 times it (probabilities
                // of up to 2^8 lose nothing in bf16 or the sums): O is hardly ever rescaled
                if (j == 0) {
                    m_run = fmaxf(cm, -FLT_MAX);  // finite: where every key so far scores -inf, probabilities of 0
                } else {
                    const bool grown = cm > m_run + grow;
                    if (__any_sync(0xffffffffu, grown)) {
                        const bool in = __all_sync(0xffffffffu, mbar_wait(odone(J - 1), ((J - 1) >> 1) & 1, a.status));  // O up to the last chunk
                        tc_fence_after();
                        const float corr = grown ? at_exp2((m_run - cm) * k2) : 1.f;
                        if (grown) m_run = cm;
                        l2[0] = mul_f32x2(l2[0], pack_f32x2(corr, corr));
                        l2[1] = mul_f32x2(l2[1], pack_f32x2(corr, corr));
#pragma unroll 1
                        for (int cb = 0; in && cb < HD; cb += 16) {
                            float ov[16];
                            uint32_t on[16];
                            tmem_ld16(t_o + cb, ov);
#pragma unroll
                            for (int u = 0; u < 16; ++u) on[u] = __float_as_uint(ov[u] * corr);
                            tmem_st16(t_o + cb, on);
                        }
                    }
                }
                const float moff = -m_run * k2;
                const uint64_t kk2 = pack_f32x2(k2, k2), mm2 = pack_f32x2(moff, moff);
#pragma unroll
                for (int b = 0; b < NK; b += 32) {
                    uint32_t pk[16];
#pragma unroll
                    for (int u = 0; u < 16; ++u) {
                        const float2 x = unpack_f32x2(fma_f32x2(pack_f32x2(v[b + 2 * u], v[b + 2 * u + 1]), kk2, mm2));
                        const float e0 = at_exp2(x.x), e1 = at_exp2(x.y);
                        pk[u] = pack_bf16(e0, e1);
                        l2[u & 1] = add_f32x2(l2[u & 1], pack_f32x2(e0, e1));
                    }
                    tmem_st16(t_s + b / 2, pk);
                }
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(pready(J));
            }
            if (ok) ok = __all_sync(0xffffffffu, mbar_wait(odone(J - 1), ((J - 1) >> 1) & 1, a.status));
            if (!ok) break;
            tc_fence_after();
            const float2 ls = unpack_f32x2(add_f32x2(l2[0], l2[1]));
            const float sum = ls.x + ls.y, inv = sum == 0.f ? 0.f : 1.f / sum;  // no key that counts: 0
            const size_t at = (((size_t)c * a.n_q + g * a.group + (live ? hr : 0)) * a.Lq + (live ? tok : 0)) * HD;
            bf16* orow = static_cast<bf16*>(a.out) + at;
            bool bad = false;
#pragma unroll
            for (int cb = 0; cb < HD; cb += 32) {
                float v[32];
                tmem_ld32(t_o + cb, v);
#pragma unroll
                for (int u = 0; u < 32; ++u) {
                    v[u] *= inv;
                    bad |= !isfinite(v[u]);
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
            if (lane == 0) mbar_arrive(oempty);
            if (live && bad) {
                const long long kv_off = (long long)(c / a.L) * a.s0 + (long long)(c % a.L) * a.s1 + (long long)g * a.s2;
#pragma unroll 1
                for (int cb = 0; cb < HD; cb += 32) {
                    float w[32];
                    row_again<bf16, HD, 32, 1>(static_cast<const bf16*>(a.Q) + at, static_cast<const bf16*>(a.K) + kv_off,
                                               static_cast<const bf16*>(a.V) + kv_off, a.s3, vis, a, cb, w);
                    for (int u = 0; u < 32; ++u) orow[cb + u] = __float2bfloat16_rn(w[u]);
                }
            }
            __syncwarp();
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == SM::MMA_WARP) tmem_dealloc(tmem, SM::TMEM);
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
    const long long tiles = (long long)((a.Lq + rows - 1) / rows) * a.n_kv * C;
    if (tiles >= 1ll << 30) return cudaErrorNotSupported;
    window_prefill_kernel<HD><<<(unsigned)std::min(tiles, 2ll * sms), WinSmem<HD>::THREADS, WinSmem<HD>::DYN, st>>>(mq, mk, mv, a, C);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_window_prefill(const AttnArgs& a, int hd, int n_ctx, int C, int sms, cudaStream_t st) {
    return hd == 64 ? launch<64>(a, n_ctx, C, sms, st) : launch<128>(a, n_ctx, C, sms, st);
}

}  // namespace mone
