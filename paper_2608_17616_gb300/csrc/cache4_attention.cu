// Attention of each context's newest tokens over its cache in 4 bits (mone_cache4_attention): the form over codes and scales.
#include "cache4_common.cuh"
#include "cache_attention.cuh"

namespace mone {

namespace {

struct Ca4Args : CaArgs {
    const uint8_t *Ks, *Vs;  // scales, strides in bytes
    long long c_layer, c_page, c_head, c_pos;
    float k_unit, v_unit;
    int near;                // 8 rows (head_dim 128) or 16 lie in a page, and its strides and its rows' have 32 bits
    int one_page;            // and a block in a page, a head's rows of it side by side
    int mask;                // of a place in its page
    long long to_v, to_vs;   // from keys to values, codes and scales
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

// ---------------------------------------------------------------- tensor cores
__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&A)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(A[0]), "r"(A[1]), "r"(A[2]), "r"(A[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_halves(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// The low half of each byte from a, the high one from b
__device__ __forceinline__ uint32_t low_or_high(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0xca;" : "=r"(r) : "r"(0x0f0f0f0fu), "r"(a), "r"(b));
    return r;
}
template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src) {
    if constexpr (BYTES == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
    else
        asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(BYTES) : "memory");
}
template <int N>
__device__ __forceinline__ void load_shared(uint32_t (&x)[N], uint32_t addr) {
    if constexpr (N == 4)
        asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(addr) : "memory");
    else if constexpr (N == 2)
        asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];" : "=r"(x[0]), "=r"(x[1]) : "r"(addr) : "memory");
    else
        asm volatile("ld.shared.b32 %0, [%1];" : "=r"(x[0]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t load_byte(uint32_t addr) {
    uint32_t x;
    asm volatile("ld.shared.u8 %0, [%1];" : "=r"(x) : "r"(addr) : "memory");
    return x;
}
__device__ __forceinline__ uint32_t load_two_bytes(uint32_t addr) {
    unsigned short x;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(x) : "r"(addr) : "memory");
    return x;
}

// A block's codes and scales come by asynchronous copies into a ring that belongs to one warp, as with the rows of 16 bits, whatever
// the strides and pages are.  The keys are the M of m16n8k16 and the rows its N, 8 or 16 of them.  Codes become halves on the way to the
// product (a conversion for two of them, a product with their scale, exact), in the lane that holds them as operands: S^T = K Q^T
// with a lane's quarter of a key's dimensions, in any order that Q has too; O^T += V^T P^T with an eighth of a value's, whose
// halves of two keys are paired by a permutation.  So nothing but the codes goes through shared memory.
//
// Halves hold a row of Q scaled by a power of two to 2^14 .. 2^15 at most (an element 2^-29 of the largest loses bits, 2^-39
// of it at most), and probabilities times 2^11, of a maximum that may since have grown by 2^4 (what is below 2^-25 of the row's
// largest loses bits, 2^-36 of it at most).  Rows of 32 bits are two halves each, 22 bits, and so are their probabilities: up to four rows (BESIDE) lie
// beside their rests in the N of 8, of more (TWO) both are multiplied one after the other.  A probability's rest is held 2^11 larger and its products add up
// apart, so that bits are lost below 2^-24 of the largest, 2^-47 of it at most (at the scale of the first halves from 2^-10 on: a row behind a large
// weight of value 0 was 2e-4 off).
// The tensor cores cut an addend off at 2^-24 of the sum and do not round it, so values of one sign came out too small by 2^-24 a product at least: 1.2e-4 after
// 65536 positions of a warp.  Of rows of 32 bits a block's products add up by themselves and then to the others', rounded, and the sum of
// the probabilities is one of what they are before their rounding (with the rests' scale, 4 layers of 131072: 118.8 us, 126.0; of more than four rows 139.1,
// 151.5).  Of rows of 16 bits, whose last bit is 2^-8, they add up in the accumulators (112.1 us for 123.6): less than 1e-4 of that length.
//
// Bound by instructions, not by HBM: 600 for a block of 32 keys of 128 (140 conversions, 128 products of halves, 34 MMAs, 32 loads from
// shared memory, 35 for the copies of a block in one page; fp32 710, with more than four rows 723; of 64 417), of which 62% of the issue slots are used, with 4 warps a scheduler and no pipe above
// half.  Two tokens over 131072 positions of 4 layers: 112 us, 604 MB at 5.4 TB/s (the rows in 16 bits: 300).  On the way: 221 us with
// masks, rescaling and a sum in every block; 175 with neither, and values' codes paired before their conversion (a permutation a pair of halves
// less); 150 with four CTAs an SM for three (128 registers a thread for 168); 136 with a piece's walk out of the registers; 119 with
// the copies of one page.  Bulk copies of a page want uniform addresses: 705 instructions, 142 for 136.  The next block's scores beside this one's
// values need 168 registers: 140, as three CTAs without.
template <typename T_, int HD_, int NT, bool BESIDE>
struct CaFour {
    using T = T_;
    static constexpr bool F32 = std::is_same<T, float>::value, TWO = F32 && !BESIDE;
    static constexpr int HD = HD_, ROWS = BESIDE ? 4 : 8 * NT, CTAS = NT == 1 ? (TWO ? 3 : 4) : 2;
    // Blocks of a warp, see item_ctas.  A second block costs a warp 0.6 us (head_dim 64) or 1, a cluster 0.9 (one layer of 370 positions 6.5 us, 7.4; with
    // three blocks a warp, two of a cluster's, 7.0 and 8.6).  With a third of the GPU's CTAs in clusters they take up to 12 blocks a warp (4 layers of
    // 9000, hd 128: 18.3 us, dealt 22.3), with fewer 6 (one of 9000: 12.3 and 11.6), with more 16 (8 contexts of up to 9000: 14.0 and 17.1).
    // A row's scales are 4 or 8 bytes of a sector of 32.  Two tokens over 131072 positions of 4 layers, heads and layers in step, heads only, neither: 112 us,
    // 117, 120; of pools whose heads lie inside positions 122, 151, 231 (1.46 GB read); head_dim 64 78, 81, 83, inside positions 87, 92, 197; 16 contexts
    // of 32K in fp32 73, 73, 80 (74 since its sums are rounded).
    static constexpr bool IN_STEP = true;
    using Walk = CaWalk<IN_STEP>;
    static constexpr int ONE = 2, EACH = 1, FULL = 16, SOME = 12, FEW = 6;
    static constexpr int CODES = KB * HD / 2, SCALES = KB * HD / 16, STAGE = 2 * (CODES + SCALES);
    static constexpr int NS = HD == 64 ? 4 : 2;  // (3 for 128: 121 us for 119, with less of the L1 left)
    // The ring, and what is not in registers while a piece's blocks go through: the walk of the copies, that of the products, the place of
    // the piece's scores and its head's addresses
    static constexpr int AHEAD = NS * STAGE, NOW = AHEAD + sizeof(Walk), SCORES = NOW + sizeof(Walk), WARP_BYTES = AHEAD + 256, ALIGN = 128;
    static constexpr int CHUNKS = HD / 32;  // of 16 bytes, of a row's codes
    // Of the probabilities and their rests (the growth that is let pass: with 2^8, and 2^7 for 2^11, 111.5 us for 112.1 and bits lost from 2^-21 on)
    static constexpr float P_LOG2 = 11.f, P_UNIT_INV = 0x1p-11f, P_ROOM = 4.f, REST = 0x1p11f, REST_INV = 0x1p-11f, FROM_NONE = -3e38f;
    static_assert(CTAS * (CA_WARPS * WARP_BYTES + ALIGN + 1536) <= 228 * 1024, "CTAs an SM");
    static_assert(Part<HD, ROWS>::FLOATS * 4 <= AHEAD, "a part fits in the ring");
    static_assert(sizeof(Walk) % 16 == 0 && SCORES + 32 <= WARP_BYTES, "what is put aside");

    using Args = Ca4Args;
    using Maps = NoMaps;
    using Head = FourHead;

    uint32_t ring, lane;
    float* ring_part;  // the ring as the place of the warp's last part
    // Places in a stage: of the codes that this lane copies, of its quarter of key gq, its eighth of values 2 t and 2 t + 1, and their
    // scales.  (Of the first eight rows; the others are at fixed distances.)
    uint32_t copy_at, key_at, val_at[2], key_scale_at, val_scale_at;

    // Byte of chunk c of row r: neighbouring rows, and for head_dim 128 halves of a row, change places so that neither the loads of
    // keys (neighbouring rows) nor those of values (every other row, the same bytes of each) meet in a bank.  Rows 8 further on
    // are 8 rows of bytes further on.
    static __device__ __forceinline__ uint32_t at(int r, int c) { return (r ^ (r >> 2 & 1)) * (HD / 2) + (HD == 128 ? c ^ (r & 2) : c) * 16; }

    __device__ CaFour(const NoMaps&, uint8_t* smem, int) : ring_part(reinterpret_cast<float*>(smem)) {
        // (kept in registers: found anew for every block they took 13 instructions of 750)
        asm volatile("mov.b32 %0, %1;" : "=r"(ring) : "r"(smem_u32(smem)));
        asm volatile("mov.u32 %0, %%laneid;" : "=r"(lane));
        const int gq = lane >> 2, t = lane & 3;
        copy_at = at(lane / CHUNKS, lane % CHUNKS);
        key_at = HD == 128 ? at(gq, t) : at(gq, 0) + 8 * t;
        for (int y = 0; y < 2; ++y) val_at[y] = CODES + (HD == 128 ? at(2 * t + y, gq >> 1) + 8 * (gq & 1) : at(2 * t + y, 0) + 4 * gq);
        key_scale_at = 2 * CODES + gq * (HD / 16) + (HD == 128 ? 2 * t : t);
        val_scale_at = 2 * CODES + SCALES + 2 * t * (HD / 16) + (HD == 128 ? gq : gq >> 1);
    }

    // The copies of a warp's blocks, ahead of their reading and on through the pieces.  A lane looks up a key's page a block ahead and
    // copies its scales, neighbours copy its codes: 8 rows with one instruction (head_dim 128) or 16.
    struct Feed {
        int left = 0, j0, page;  // blocks of the piece (-1: no more pieces); the first key of the next, the lane's key's page
        int gap;                 // the end of the first positions' blocks
    };
    // A walk put aside, by every lane the same, and back
    __device__ __forceinline__ void put(int at, const Walk& w) const {
        const uint4* u = reinterpret_cast<const uint4*>(&w);
#pragma unroll
        for (int i = 0; i < (int)sizeof(Walk) / 16; ++i)
            asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(ring + at + 16 * i), "r"(u[i].x), "r"(u[i].y), "r"(u[i].z), "r"(u[i].w) : "memory");
    }
    __device__ __forceinline__ void get(int at, Walk& w) const {
        uint4* u = reinterpret_cast<uint4*>(&w);
#pragma unroll
        for (int i = 0; i < (int)sizeof(Walk) / 16; ++i)
            asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(u[i].x), "=r"(u[i].y), "=r"(u[i].z), "=r"(u[i].w) : "r"(ring + at + 16 * i) : "memory");
    }
    __device__ __forceinline__ int aside(int at) const {
        int x;
        asm volatile("ld.shared.b32 %0, [%1];" : "=r"(x) : "r"(ring + at) : "memory");
        return x;
    }
    __device__ __forceinline__ void put_pointer(int at, const void* p) const { asm volatile("st.shared.b64 [%0], %1;" ::"r"(ring + at), "l"(p) : "memory"); }
    template <typename P>
    __device__ __forceinline__ const P* pointer(int at) const {
        const P* p;
        asm volatile("ld.shared.b64 %0, [%1];" : "=l"(p) : "r"(ring + at) : "memory");
        return p;
    }
    static constexpr int R_N = offsetof(Walk, r) + offsetof(CaRange, n), R_T0 = offsetof(Walk, r) + offsetof(CaRange, t0),
                         R_LO = offsetof(Walk, r) + offsetof(CaRange, lo);
    // The first block of a walk's next piece that has any
    __device__ __forceinline__ void begin(const Args& a, Feed& f, Walk& w) const {
        do {
            if (!w.next(a)) {
                f.left = -1;
                return;
            }
            f.left = w.b1 - w.b0;
        } while (f.left == 0);
        put(AHEAD, w);
        f.gap = w.r.ns * KB;
        f.j0 = w.r.at(w.b0);
        const FourHead head(a, w.l, w.g);
        // (V is as far from K in every head)
        put_pointer(SCORES + 8, head.K);
        put_pointer(SCORES + 16, head.Ks);
        put_pointer(SCORES + 24, a.v.table + (size_t)w.c * a.v.width);
        page(a, f, w.r.n, w.r.t0);
    }
    __device__ __forceinline__ void page(const Args& a, Feed& f, int n, int t0) const {
        const int key = f.j0 + lane;
        f.page = key < n && (key < a.n_sink || key > t0 - a.window) ? pointer<int>(SCORES + 24)[key >> a.v.page_log2] : INT_MIN;
    }
    __device__ __forceinline__ void look(const Args& a, Feed& f) const {
        if (f.left) {
            f.j0 += KB;
            if (f.j0 == f.gap) f.j0 = aside(AHEAD + R_LO);
            page(a, f, aside(AHEAD + R_N), aside(AHEAD + R_T0));
        } else {
            Walk w;
            get(AHEAD, w);
            __syncwarp();
            begin(a, f, w);
        }
    }
    __device__ __forceinline__ void feed(const Args& a, Feed& f, int s) {
        constexpr int R = 32 / CHUNKS;  // rows of an instruction
        if (f.left >= 0) {
            const uint8_t *K = pointer<uint8_t>(SCORES + 8) + 16 * (lane % CHUNKS), *Ks = pointer<uint8_t>(SCORES + 16);
            const uint32_t dst = ring + s * STAGE + copy_at, scales = ring + s * STAGE + 2 * CODES + lane * (HD / 16);
            if (__builtin_expect(a.near && __all_sync(0xffffffffu, (unsigned)f.page < (unsigned)a.v.n_pages), 1)) {  // all are there
                if (a.one_page) {  // (35 instructions of a block's 600 for 75)
                    const unsigned row = f.j0 & a.mask;
                    const uint8_t* ks = Ks + (unsigned long long)f.page * (unsigned)a.c_page + (row + lane) * (HD / 16);
                    copy_async<HD / 16>(scales, ks);
                    copy_async<HD / 16>(scales + SCALES, ks + a.to_vs);
                    const uint8_t *k = K + (unsigned long long)f.page * (unsigned)a.v.s_page + (row * (HD / 2) + lane / CHUNKS * (HD / 2)), *v = k + a.to_v;
#pragma unroll
                    for (int x = 0; x < CHUNKS; ++x) {
                        copy_async<16>(dst + x * R * (HD / 2), k + x * R * (HD / 2));
                        copy_async<16>(dst + x * R * (HD / 2) + CODES, v + x * R * (HD / 2));
                    }
                } else {
                    auto place = [&](unsigned page, unsigned row, long long s_page, long long s_pos) {
                        return (unsigned long long)page * (unsigned)s_page + (unsigned long long)row * (unsigned)s_pos;
                    };
                    const uint8_t* ks = Ks + place(f.page, (f.j0 + lane) & a.mask, a.c_page, a.c_pos);
                    copy_async<HD / 16>(scales, ks);
                    copy_async<HD / 16>(scales + SCALES, ks + a.to_vs);
#pragma unroll
                    for (int x = 0; x < CHUNKS; ++x) {
                        const uint8_t* k = K + place(__shfl_sync(0xffffffffu, f.page, x * R), ((f.j0 + x * R) & a.mask) + lane / CHUNKS, a.v.s_page, a.v.s_pos);
                        copy_async<16>(dst + x * R * (HD / 2), k);
                        copy_async<16>(dst + x * R * (HD / 2) + CODES, k + a.to_v);
                    }
                }
            } else {
                bool in = f.page != INT_MIN;
                if (in && (unsigned)f.page >= (unsigned)a.v.n_pages) {
                    cache_fail(a.v.status, DS_CACHE_PAGE);
                    in = false;
                }
                const int row = (f.j0 + lane) & a.mask;
                if (in) {
                    const uint8_t* ks = Ks + (f.page * a.c_page + row * a.c_pos);
                    copy_async<HD / 16>(scales, ks);
                    copy_async<HD / 16>(scales + SCALES, ks + a.to_vs);
                }
                const long long mine = in ? f.page * a.v.s_page + row * a.v.s_pos : -1;
#pragma unroll 1
                for (int x = 0; x < CHUNKS; ++x) {
                    const long long off = __shfl_sync(0xffffffffu, mine, x * R + lane / CHUNKS);
                    if (off < 0) continue;
                    copy_async<16>(dst + x * R * (HD / 2), K + off);
                    copy_async<16>(dst + x * R * (HD / 2) + CODES, K + off + a.to_v);
                }
            }
            --f.left;
            look(a, f);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }

    // A warp's rows of an item and what it has of them.  Lane 4 gq + t has a quarter of Q of row 8 i + gq, dimensions from t HD / 4; S
    // and the sums of rows 8 i + 2 t and + 1, and of these O's dimensions gq HD / 8 + 2 m (0, 1) and + 1 (2, 3).  (BESIDE: of row
    // gq % 4, if gq >= 4 its rest; of rows 2 (t % 2) and + 1, if t >= 2 what their rests give to O.)
    struct Rows {
        uint32_t q[TWO ? 2 : 1][NT][HD / 16][2];
        float o[NT][HD / 16][4];
        float l[F32 ? 1 : NT][4];      // the sums of the probabilities that O's products see, in the layout of O (each twice); not F32
        float lx[NT][2];               // of the exact ones, this lane's: F32, or with scores
        float from[NT][2];             // what is taken off a row's S: within P_ROOM of its maximum in base 2, or FROM_NONE
        float unit[NT], k2[NT][2];     // of S: the unit in which it is q k (of row 8 i + gq), and in base 2 with the softmax's scale
    };

    static __device__ __forceinline__ void add(float (&d)[4], const float (&x)[4], float unit) {
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
            const float2 a = make_float2(x[i], x[i + 1]), b = make_float2(d[i], d[i + 1]);
            const float2 s = unit == 1.f ? add2(a, b) : fma2(a, make_float2(unit, unit), b);
            d[i] = s.x;
            d[i + 1] = s.y;
        }
    }

    // the row of h = 0, 1
    __device__ __forceinline__ int row_of(int i, int h) const { return BESIDE ? 2 * (lane & 1) + h : 8 * i + 2 * (lane & 3) + h; }

    // Q of row `row` of all, this lane's quarter, and the power of two that it is to be multiplied with
    __device__ __forceinline__ float load_q(const Args& a, size_t row, bool live, uint32_t (&hi)[HD / 16][2], uint32_t (*lo)[2]) const {
        constexpr int D = HD / 4, PER = 16 / sizeof(T);
        const int t = lane & 3;
        const T* q = static_cast<const T*>(a.Q) + row * HD + t * D;
        float x[D], most = 0.f;
#pragma unroll
        for (int p = 0; p < D / PER; ++p) {
            const uint4 u = live ? reinterpret_cast<const uint4*>(q)[p] : make_uint4(0, 0, 0, 0);
            const T* e = reinterpret_cast<const T*>(&u);
#pragma unroll
            for (int i = 0; i < PER; ++i) x[p * PER + i] = to_f<T>(e[i]);
        }
#pragma unroll
        for (int i = 0; i < D; ++i) most = fmaxf(most, isnan(x[i]) ? INFINITY : fabsf(x[i]));
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
        const int e = max((int)(__float_as_uint(most) >> 23), 16);
        float scale = __uint_as_float((unsigned)(268 - e) << 23), unit = __uint_as_float((unsigned)(e - 14) << 23);
        const bool finite = most < INFINITY;
        if (!finite) scale = unit = 1.f;
#pragma unroll
        for (int i = 0; i < D; i += 2) {
            // beside an infinity or a NaN, what is finite has no say
            const float x0 = finite || !isfinite(x[i]) ? x[i] * scale : 0.f, x1 = finite || !isfinite(x[i + 1]) ? x[i + 1] * scale : 0.f;
            const uint32_t h = pack_halves(x0, x1);
            hi[i / 4][i / 2 % 2] = h;
            if constexpr (TWO || BESIDE) {
                const float2 f = halves_float2(h);
                const uint32_t rest = finite ? pack_halves(x0 - f.x, x1 - f.y) : 0;
                if constexpr (TWO)
                    lo[i / 4][i / 2 % 2] = rest;
                else if (lane >= 16)
                    hi[i / 4][i / 2 % 2] = rest;
            }
        }
        return unit;
    }

    __device__ __forceinline__ void run(const Args& a, CaNote* notes) {
        using P = Part<HD, ROWS>;
        const int gq = lane >> 2, t = lane & 3;
        const float scale2 = a.scale * 1.4426950408889634f;
        Walk w(a);
        Feed ahead;
        int slot = 0;  // of the block to be read next
        {
            Walk first = w;
            begin(a, ahead, first);
        }
#pragma unroll 1
        for (int s = 0; s < NS - 1; ++s) feed(a, ahead, s);
        while (w.next(a)) {
            const int row0 = w.rt * ROWS, rows = min(ROWS, a.R - row0);
            put(NOW, w);
            if (a.z2) asm volatile("st.shared.b64 [%0], %1;" ::"r"(ring + SCORES), "l"(a.z2 + (w.kv(a) * a.R + row0) * a.pitch) : "memory");
            Rows x;
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                const int q_row = BESIDE ? gq & 3 : 8 * i + gq;
                const bool live = q_row < rows;
                x.unit[i] = load_q(a, w.kv(a) * a.R + row0 + (live ? q_row : 0), live, x.q[0][i], TWO ? x.q[TWO][i] : nullptr) * a.k_unit;
#pragma unroll
                for (int k = 0; k < HD / 16; ++k) x.o[i][k][0] = x.o[i][k][1] = x.o[i][k][2] = x.o[i][k][3] = 0.f;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int row = row_of(i, h);
                    x.from[i][h] = FROM_NONE;
                    if constexpr (!F32) x.l[i][h] = x.l[i][2 + h] = 0.f;
                    x.lx[i][h] = 0.f;
                    const float k2 = scale2 * __shfl_sync(0xffffffffu, x.unit[i], 4 * (row - 8 * i));
                    x.k2[i][h] = fminf(fmaxf(k2, 1e-37f), 1e38f);  // (0 and infinity would make 0 of nothing)
                }
            }
            int j0 = w.r.at(w.b0);
            const int gap = w.r.ns * KB;
            // blocks that every row sees whole: from here on, and within the first positions, up to there
            const int whole0 = w.r.n - a.window, whole1 = w.r.n - a.n_tok + 1 - KB;
#pragma unroll 1
            for (int left = w.b1 - w.b0; left > 0; --left) {
                asm volatile("cp.async.wait_group %0;" ::"n"(NS - 2) : "memory");
                __syncwarp();
                feed(a, ahead, slot == 0 ? NS - 1 : slot - 1);  // into the slot that was read last
                if (__builtin_expect(j0 <= whole1 && (j0 >= whole0 || j0 + KB <= a.n_sink), 1))
                    step<true>(a, j0, slot, rows, x);
                else
                    step<false>(a, j0, slot, rows, x);
                __syncwarp();  // the block has been read
                if (++slot == NS) slot = 0;
                j0 += KB;
                if (j0 == gap) j0 = aside(NOW + R_LO);
            }
            get(NOW, w);
            __syncwarp();
            const size_t kv = w.kv(a);
            // a part goes to the workspace while the ring is in use
            float* part = w.last ? ring_part : P::of_warp(a, w.b0 == 0);
            if (w.whole && lane == 0) a.info[kv * a.RT + w.rt] = 1 << 16;
            if (!w.whole && lane == 0) notes[w.b0 == 0] = {part, w.c, w.l, w.g, w.rt, w.r.n, w.first, w.cta_whole, w.parts};
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float lx = x.lx[i][h] * P_UNIT_INV;
#pragma unroll
                    for (int y = 4; y < 32; y <<= 1) lx += __shfl_xor_sync(0xffffffffu, lx, y);
                    const float l = F32 ? lx : x.l[i][h] * P_UNIT_INV;
                    const int row = row_of(i, h), d0 = gq * (HD / 8);
                    const float unit = __shfl_sync(0xffffffffu, x.unit[i], 4 * (row - 8 * i));
                    float v[HD / 8];
#pragma unroll
                    for (int d = 0; d < HD / 8; ++d) v[d] = x.o[i][d / 2][d % 2 * 2 + h] * P_UNIT_INV;
                    if constexpr (BESIDE) {
#pragma unroll
                        for (int d = 0; d < HD / 8; ++d) v[d] = fmaf(__shfl_xor_sync(0xffffffffu, v[d], 2), REST_INV, v[d]);
                    }
                    if (row >= rows || (BESIDE && t >= 2)) continue;
#pragma unroll
                    for (int d = 0; d < HD / 8; ++d) v[d] *= a.v_unit;
                    const float m = x.from[i][h] == FROM_NONE ? -INFINITY : x.from[i][h] * unit;
                    if (w.whole) {
                        finish_row<CaFour, HD / 8>(a, kv, w.c, w.l, w.g, w.r.n, w.rt * ROWS + row, d0, v, l);
                        T* out = static_cast<T*>(a.out) + (kv * a.R + w.rt * ROWS + row) * HD + d0;
                        __align__(16) T y[HD / 8];
#pragma unroll
                        for (int d = 0; d < HD / 8; ++d) y[d] = from_f<T>(v[d]);
#pragma unroll
                        for (int d = 0; d < (int)(HD / 8 * sizeof(T) / 16); ++d) reinterpret_cast<uint4*>(out)[d] = reinterpret_cast<const uint4*>(y)[d];
                        if (gq == 0 && a.lse) a.lse[kv * a.R + w.rt * ROWS + row] = row_lse(m, lx, scale2);
                    } else {
#pragma unroll
                        for (int d = 0; d < HD / 8; d += 4)
                            *reinterpret_cast<float4*>(part + row * HD + d0 + d) = make_float4(v[d], v[d + 1], v[d + 2], v[d + 3]);
                        if (gq == 0) {
                            part[P::M + row] = m;
                            part[P::L + row] = l;
                            part[P::LX + row] = lx;
                        }
                    }
                }
            __syncwarp();
        }
    }

    // One block's keys; WHOLE: every row sees all of them
    template <bool WHOLE>
    __device__ __forceinline__ void step(const Args& a, int j0, int slot, int rows, Rows& x) {
        const int gq = lane >> 2, t = lane & 3;
        const uint32_t stage = ring + slot * STAGE;
        const int n = WHOLE ? 0 : aside(NOW + R_N), t0 = WHOLE ? 0 : aside(NOW + R_T0);
        float s[NT][2][4];  // of keys 16 u + gq (0, 1) and + 8 (2, 3), rows 2 t and + 1
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
            for (int i = 0; i < NT; ++i) s[i][u][0] = s[i][u][1] = s[i][u][2] = s[i][u][3] = 0.f;
            uint32_t w[2][HD / 32], sc[2][HD / 64];
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const int row = 16 * u + 8 * y;  // and gq
                load_shared(w[y], stage + key_at + row * (HD / 2));
                if constexpr (HD == 128) {
                    const uint32_t two = scale_halves(load_two_bytes(stage + key_scale_at + row * 8));
                    sc[y][0] = __byte_perm(two, 0, 0x1010);
                    sc[y][1] = __byte_perm(two, 0, 0x3232);
                } else {
                    sc[y][0] = scale_halves(load_byte(stage + key_scale_at + row * 4) * 0x101);
                }
            }
#pragma unroll
            for (int k = 0; k < HD / 32; ++k) {
                uint32_t h[2][4];
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    code_halves(w[y][k], h[y]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) h[y][e] = mul_halves(h[y][e], sc[y][k / 2]);
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t A[4] = {h[0][2 * e], h[1][2 * e], h[0][2 * e + 1], h[1][2 * e + 1]};
#pragma unroll
                    for (int i = 0; i < NT; ++i)
#pragma unroll
                        for (int y = 0; y < (TWO ? 2 : 1); ++y) mma_f16(s[i][u], A, x.q[y][i][2 * k + e][0], x.q[y][i][2 * k + e][1]);
                }
            }
        }
        if constexpr (BESIDE) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[0][u][e] += __shfl_xor_sync(0xffffffffu, s[0][u][e], 2);
        }
        uint32_t pb[TWO ? 2 : 1][NT][2][2];  // P^T: keys 16 u + 2 t, + 1 (and + 8) of row gq
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            if (!WHOLE) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int row = row_of(i, h), vis = n - a.n_tok + (a.n_tok == 1 ? 0 : (aside(NOW + offsetof(Walk, rt)) * ROWS + row) % a.n_tok) + 1;
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int e = h; e < 4; e += 2) {
                            const int key = j0 + 16 * u + gq + 8 * (e >> 1);
                            s[i][u][e] = row < rows && key < vis && (key < a.n_sink || key >= vis - a.window) ? s[i][u][e] : -INFINITY;
                        }
                }
            }
            // A row whose scores have grown by more than 2^8 (its first ones) is rescaled
            float most[2];
            bool grown = false;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                most[h] = fmaxf(fmaxf(s[i][0][h], s[i][0][2 + h]), fmaxf(s[i][1][h], s[i][1][2 + h]));
                grown |= (most[h] - x.from[i][h]) * x.k2[i][h] > P_ROOM;
            }
            if (__any_sync(0xffffffffu, grown)) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
#pragma unroll
                    for (int y = 4; y < 32; y <<= 1) most[h] = fmaxf(most[h], __shfl_xor_sync(0xffffffffu, most[h], y));
                    // (by its own scores alone, whatever the item's other rows are)
                    const float to = (most[h] - x.from[i][h]) * x.k2[i][h] > P_ROOM ? most[h] : x.from[i][h];
                    const float f = ca_exp2((x.from[i][h] - to) * x.k2[i][h]);
                    x.from[i][h] = to;
                    x.lx[i][h] *= f;
                    if constexpr (!F32) x.l[i][h] *= f;
#pragma unroll
                    for (int d = 0; d < HD / 16; ++d) {
                        x.o[i][d][h] *= f;
                        x.o[i][d][2 + h] *= f;
                    }
                }
            }
            float e[2][4];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int k = 0; k < 4; ++k) e[u][k] = ca_exp2(fmaf(s[i][u][k] - x.from[i][k & 1], x.k2[i][k & 1], P_LOG2));
            if (F32 || a.z2) {
#pragma unroll
                for (int h = 0; h < 2; ++h) x.lx[i][h] += (e[0][h] + e[0][2 + h]) + (e[1][h] + e[1][2 + h]);
            }
            if (a.z2) {
                float* z0;
                asm volatile("ld.shared.b64 %0, [%1];" : "=l"(z0) : "r"(ring + SCORES) : "memory");
                z0 += j0 + gq;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (row_of(i, h) < rows && !(BESIDE && t >= 2)) {
                        float* z = z0 + row_of(i, h) * a.pitch;
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            z[16 * u] = s[i][u][h] * x.k2[i][h];
                            z[16 * u + 8] = s[i][u][2 + h] * x.k2[i][h];
                        }
                    }
                }
            }
            const uint32_t ones[4] = {0x3c003c00u, 0x3c003c00u, 0x3c003c00u, 0x3c003c00u};
#pragma unroll
            for (int u = 0; u < 2; ++u) {
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    uint32_t p = pack_halves(e[u][2 * half], e[u][2 * half + 1]);
                    if constexpr (F32) {
                        const float2 f = fma2(halves_float2(p), make_float2(-REST, -REST),
                                              mul2(make_float2(e[u][2 * half], e[u][2 * half + 1]), make_float2(REST, REST)));
                        const uint32_t rest = pack_halves(f.x, f.y);
                        if constexpr (TWO)
                            pb[TWO][i][u][half] = ca_transpose(rest);
                        else
                            p = t >= 2 ? rest : p;
                    }
                    pb[0][i][u][half] = ca_transpose(p);
                }
                if constexpr (!F32) mma_f16(x.l[i], ones, pb[0][i][u][0], pb[0][i][u][1]);
            }
        }
        uint32_t w[F32 ? 2 : 1][4][HD / 64], sc[F32 ? 2 : 1][2];
        auto load = [&](int u, uint32_t (&w)[4][HD / 64], uint32_t (&sc)[2]) {
            uint32_t b[4];
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const int row = 16 * u + 8 * (y >> 1);  // and 2 t, and 1
                load_shared(w[y], stage + val_at[y & 1] + row * (HD / 2));
                b[y] = load_byte(stage + val_scale_at + (row + (y & 1)) * (HD / 16));
                if (!WHOLE) {  // a scale that no row sees is not to meet a probability of 0
                    const int j = j0 + row + 2 * t + (y & 1);
                    b[y] = j < n && (j < a.n_sink || j > t0 - a.window) ? b[y] : 0;
                }
            }
            sc[0] = scale_halves(b[0] | b[1] << 8);
            sc[1] = scale_halves(b[2] | b[3] << 8);
        };
        auto product = [&](int u, int k, const uint32_t (&w)[4][HD / 64], const uint32_t (&sc)[2], float (&sum)[F32 ? 4 : 1][4], float (&rest)[TWO ? 4 : 1][4]) {
            uint32_t h[2][2][4];  // of keys 2 t and + 1 (and + 8), elements 8 k + 2 e and + 1: a code of either in a byte
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const uint32_t p = w[2 * y][k], q = w[2 * y + 1][k];
                code_halves(low_or_high(p, q << 4), h[y][0]);
                code_halves(low_or_high(p >> 4, q), h[y][1]);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                uint32_t A[4];
#pragma unroll
                for (int y = 0; y < 4; ++y) A[y] = mul_halves(h[y >> 1][y & 1][e], sc[y >> 1]);
#pragma unroll
                for (int i = 0; i < NT; ++i) mma_f16(F32 ? sum[F32 ? e : 0] : x.o[i][4 * k + e], A, pb[0][i][u][0], pb[0][i][u][1]);
                if constexpr (TWO) mma_f16(rest[e], A, pb[TWO][0][u][0], pb[TWO][0][u][1]);
            }
        };
        if constexpr (F32) {
            load(0, w[0], sc[0]);
            load(1, w[F32], sc[F32]);
#pragma unroll
            for (int k = 0; k < HD / 64; ++k) {
                float sum[4][4] = {}, rest[TWO ? 4 : 1][4] = {};
                product(0, k, w[0], sc[0], sum, rest);
                product(1, k, w[F32], sc[F32], sum, rest);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    add(x.o[0][4 * k + e], sum[e], 1.f);
                    if constexpr (TWO) add(x.o[0][4 * k + e], rest[e], REST_INV);
                }
            }
        } else {
            float none[1][4];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                load(u, w[0], sc[0]);
#pragma unroll
                for (int k = 0; k < HD / 64; ++k) product(u, k, w[0], sc[0], none, none);
            }
        }
    }
};

template <int HD>
cudaError_t launch_four(const DevState& s, const Ca4Args& a, int* kernels, cudaStream_t st) {
    if (s.dtype == 0)
        return a.R <= 4 ? launch<CaFour<float, HD, 1, true>>(a, {}, s.sms, kernels, st) : launch<CaFour<float, HD, 1, false>>(a, {}, s.sms, kernels, st);
    return a.R <= 8 ? launch<CaFour<bf16, HD, 1, false>>(a, {}, s.sms, kernels, st) : launch<CaFour<bf16, HD, 2, false>>(a, {}, s.sms, kernels, st);
}

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
    a.near = f.v.page_log2 >= (s.hd == 64 ? 4 : 3) && std::max({f.v.s_page, f.v.s_pos, f.c_page, f.c_pos}) < 1ll << 32;
    a.one_page = a.near && f.v.page_log2 >= 5 && f.v.s_pos == s.hd / 2 && f.c_pos == s.hd / 16;
    a.mask = (1 << f.v.page_log2) - 1;
    a.to_v = static_cast<const uint8_t*>(f.v.V) - static_cast<const uint8_t*>(f.v.K);
    a.to_vs = f.Vs - f.Ks;
    return s.hd == 64 ? launch_four<64>(s, a, kernels, st) : launch_four<128>(s, a, kernels, st);
}

}  // namespace mone
