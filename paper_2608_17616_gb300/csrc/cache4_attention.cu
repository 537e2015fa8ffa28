// Attention of each context's newest tokens over its cache in 4 bits (mone_cache4_attention): the form over codes and scales.
#include "cache4_common.cuh"
#include "cache_attention.cuh"

namespace mone {

namespace {

struct Ca4Args : CaArgs {
    const uint8_t *Ks, *Vs;  // scales, strides in bytes
    long long c_layer, c_page, c_head, c_pos;
    float k_unit, v_unit;
};

struct FourHead {
    const uint8_t *K, *V, *Ks, *Vs;
    long long s_page, s_pos, c_page, c_pos;
    float k_unit, v_unit;
    struct Row {
        const uint8_t *K, *V, *Ks, *Vs;
        float k_unit, v_unit;
        static __device__ float at(const uint8_t* codes, const uint8_t* scales, int d, float unit) {
            uint32_t h[4];
            code_halves(codes[d >> 1] >> (4 * (d & 1)) & 15, h);
            return halves_float2(h[0]).x * scale_float(scales[d >> 4]) * unit;
        }
        __device__ float k(int d) const { return at(K, Ks, d, k_unit); }
        __device__ float v(int d) const { return at(V, Vs, d, v_unit); }
    };
    __device__ FourHead(const Ca4Args& a, int l, int g)
        : s_page(a.v.s_page), s_pos(a.v.s_pos), c_page(a.c_page), c_pos(a.c_pos), k_unit(a.k_unit), v_unit(a.v_unit) {
        const long long code = l * a.v.s_layer + g * a.v.s_head, scale = l * a.c_layer + g * a.c_head;
        K = static_cast<const uint8_t*>(a.v.K) + code;
        V = static_cast<const uint8_t*>(a.v.V) + code;
        Ks = a.Ks + scale;
        Vs = a.Vs + scale;
    }
    __device__ Row row(int page, int place) const {
        const long long code = page * s_page + place * s_pos, scale = page * c_page + place * c_pos;
        return {K + code, V + code, Ks + scale, Vs + scale, k_unit, v_unit};
    }
};

// ---------------------------------------------------------------- CUDA cores
// Eight lanes share a key, each with head_dim / 8 neighbouring dimensions; the four lane groups of a warp take every fourth key and
// keep a softmax of their own, joined at the end of the piece.
template <typename T_, int HD_>
struct CaFour {
    using T = T_;
    static constexpr int HD = HD_, ROWS = 4, CTAS = HD == 64 ? 3 : 2;
    static constexpr int D = HD / 8;  // dimensions of a lane
    static constexpr int ONE = 1, EACH = 1, FULL = 1, FEW = 1;  // blocks of a warp, see item_ctas
    static constexpr int WARP_BYTES = 2 * Part<HD, ROWS>::FLOATS * 4;
    using Args = Ca4Args;
    using Maps = NoMaps;
    using Head = FourHead;

    float* parts;

    __device__ CaFour(const NoMaps&, uint8_t* smem, int) : parts(reinterpret_cast<float*>(smem)) {}

    __device__ __forceinline__ void run(const Args& a, CaNote* notes) {
        CaWalk walk(a);
        while (walk.next(a)) piece(a, walk, notes);
    }

    static __device__ __forceinline__ void decode(const uint8_t* codes, const uint8_t* scales, bool in, int l8, float unit, float (&f)[D]) {
#pragma unroll
        for (int d = 0; d < D; ++d) f[d] = 0.f;
        if (!in) return;
        const float s = scale_float(scales[l8 * D / 16]) * unit;
#pragma unroll
        for (int w = 0; w < D / 8; ++w) {
            uint32_t h[4];
            code_halves(*reinterpret_cast<const uint32_t*>(codes + l8 * D / 2 + 4 * w), h);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 two = halves_float2(h[i]);
                f[8 * w + 2 * i] = two.x * s;
                f[8 * w + 2 * i + 1] = two.y * s;
            }
        }
    }

    __device__ __forceinline__ void piece(const Args& a, const CaWalk& walk, CaNote* notes) {
        const CaRange& r = walk.r;
        const int c = walk.c, row0 = walk.rt * ROWS, rows = min(ROWS, a.R - row0);
        const size_t kv = walk.kv(a);
        const Head head(a, walk.l, walk.g);
        const float k2 = a.scale * 1.4426950408889634f;
        const int lane = threadIdx.x & 31, grp = lane >> 3, l8 = lane & 7;
        const int* table = a.v.table + (size_t)c * a.v.width;
        const int mask = (1 << a.v.page_log2) - 1;
        float q[ROWS][D], o[ROWS][D], m[ROWS], l[ROWS];
        int vis[ROWS];
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const int row = row0 + min(i, rows - 1);
            const T* qr = static_cast<const T*>(a.Q) + (kv * a.R + row) * HD + l8 * D;
#pragma unroll
            for (int d = 0; d < D; ++d) q[i][d] = i < rows ? to_f<T>(qr[d]) : 0.f;
            vis[i] = i < rows ? r.n - a.n_tok + row % a.n_tok + 1 : 0;
            m[i] = -INFINITY;
            l[i] = 0.f;
#pragma unroll
            for (int d = 0; d < D; ++d) o[i][d] = 0.f;
        }
        for (int b = walk.b0; b < walk.b1; ++b) {
            const int j0 = r.at(b);
#pragma unroll 1
            for (int it = 0; it < KB / 4; ++it) {
                const int key = j0 + grp + 4 * it;
                bool in = key < r.n && (key < a.n_sink || key > r.t0 - a.window);
                int page = 0;
                if (in) {
                    page = cache_page(a.v, table, key >> a.v.page_log2);
                    in = page >= 0;
                }
                float k[D], v[D];
                const auto row = head.row(max(page, 0), key & mask);
                decode(row.K, row.Ks, in, l8, a.k_unit, k);
                decode(row.V, row.Vs, in, l8, a.v_unit, v);
                float mine = 0.f;
#pragma unroll
                for (int i = 0; i < ROWS; ++i) {
                    float s = 0.f;
#pragma unroll
                    for (int d = 0; d < D; ++d) s = fmaf(q[i][d], k[d], s);
#pragma unroll
                    for (int x = 4; x > 0; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
                    const float z = in && key < vis[i] && (key < a.n_sink || key >= vis[i] - a.window) ? s : -INFINITY;
                    mine = l8 == i ? z : mine;
                    const float mn = fmaxf(m[i], z);
                    const float corr = mn == -INFINITY ? 1.f : ca_exp2((m[i] - mn) * k2), moff = mn == -INFINITY ? 0.f : -mn * k2;
                    m[i] = mn;
                    const float p = ca_exp2(fmaf(z, k2, moff));
                    l[i] = fmaf(l[i], corr, p);
#pragma unroll
                    for (int d = 0; d < D; ++d) o[i][d] = fmaf(p, v[d], o[i][d] * corr);
                }
                if (a.z2 && l8 < rows && key < r.n) a.z2[(kv * a.R + row0 + l8) * a.pitch + key] = mine * k2;
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
                const int dim = l8 * D + d;
                if (grp != i) continue;
                if (walk.whole)
                    write_row<CaFour>(a, kv, c, r.n, row0 + i, dim, head, x[0], x[1], l[i]);
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

}  // namespace

size_t cache4_attention_workspace(const DevState& s, const Cache4View& f, int n_q, int n_tok) {
    const long long tiles = (n_q / f.v.n_kv * n_tok + 3) / 4;  // as mone_cache_attention counts them
    if (max_blocks(f.v) * f.v.n_ctx * f.v.L * f.v.n_kv * tiles >= 1 << 30) return 0;
    return Layout(s, f.v, n_q, n_tok).bytes;
}

cudaError_t launch_cache4_attention(const DevState& s, const Cache4View& f, const void* Q, int n_q, int n_tok, int n_sink, int window, void* out,
                                    void* ws, int* kernels, cudaStream_t st) {
    Ca4Args a{};
    ca_common(a, s, f.v, Layout(s, f.v, n_q, n_tok), Q, n_q, n_tok, n_sink, window, out, ws);
    a.Ks = f.Ks; a.Vs = f.Vs;
    a.c_layer = f.c_layer; a.c_page = f.c_page; a.c_head = f.c_head; a.c_pos = f.c_pos;
    a.k_unit = f.k_unit; a.v_unit = f.v_unit;
    if (s.dtype == 0) return s.hd == 64 ? launch<CaFour<float, 64>>(a, {}, s.sms, kernels, st) : launch<CaFour<float, 128>>(a, {}, s.sms, kernels, st);
    return s.hd == 64 ? launch<CaFour<bf16, 64>>(a, {}, s.sms, kernels, st) : launch<CaFour<bf16, 128>>(a, {}, s.sms, kernels, st);
}

}  // namespace mone
