// Queries and keys normalised by head and rotated by position, in one pass (mone_norm_rotate).
#include <algorithm>
#include <climits>
#include <type_traits>

#include "mone_common.cuh"

namespace mone {

namespace {

constexpr int NR_THREADS = 128;
constexpr int NR_DEPTH = 4;           // rows under way, one of them being computed
constexpr int NR_CHUNK = 16;          // rows of a job, at most
constexpr int NR_FILL = 152 * 1024;   // threads that a launch keeps, if it has them

struct NormRotateArgs {
    RotateArgs r;
    int rows, chunk;  // rows of a token (every layer, every head of both sides); of them, those of a job
    long long jobs;
};

// cos and sin of an angle of `turn` 2^-64ths of a whole turn.  The nearest quarter turn is taken off exactly; the angle that is left,
// an eighth of a turn at most, is off by 2^-23 of itself at most, however small it is: the nearest multiple of 2^-32 turns and what is left to it, of
// either sign, are each rounded to 24 bits.
__device__ __forceinline__ void cos_sin(unsigned long long turn, float& c, float& s) {
    const int32_t lo = (int32_t)(uint32_t)turn;
    const uint32_t hi = (uint32_t)(turn >> 32) + ((uint32_t)turn >> 31);
    const uint32_t quarter = (hi + 0x20000000u) >> 30;
    const int32_t rest = (int32_t)(hi - (quarter << 30));
    float x, y;
    sincospif(fmaf((float)lo, 0x1p-63f, (float)rest * 0x1p-31f), &y, &x);
    c = quarter & 1 ? -y : x;
    s = quarter & 1 ? x : y;
    if (quarter & 2) {
        c = -c;
        s = -s;
    }
}

// What a lane has of a row, 16 elements: NP chunks of 16 bytes, neighbouring lanes' beside one another
template <typename T>
struct Chunks {
    static constexpr int E = 16 / sizeof(T), NP = 16 / E, H = NP / 2, F = E / 2;  // elements; chunks, half of them; pairs of elements of a chunk
};

// Rows under way: a lane's chunks, in shared memory at a place of its own, so that it waits for nobody else.
template <typename T, bool VEC>
struct Ring : Chunks<T> {
    using Chunks<T>::E;
    using Chunks<T>::NP;
    using Chunks<T>::F;
    static constexpr int BYTES = NR_DEPTH * NP * 16 * NR_THREADS;
    uint8_t* at;
    __device__ __forceinline__ explicit Ring(uint8_t* smem) : at(smem + 16 * threadIdx.x) {}
    __device__ __forceinline__ uint4* place(int slot, int k) const { return reinterpret_cast<uint4*>(at + (slot * NP + k) * 16 * NR_THREADS); }
    __device__ __forceinline__ void copy(int slot, const T* row, const int (&d)[NP]) const {
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            if constexpr (VEC) {
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(place(slot, k))), "l"(row + d[k]) : "memory");
            } else {
                __align__(16) T t[E];
#pragma unroll
                for (int i = 0; i < E; ++i) t[i] = row[d[k] + i];
                *place(slot, k) = *reinterpret_cast<const uint4*>(t);
            }
        }
    }
    // in pairs, chunk after chunk
    __device__ __forceinline__ void read(int slot, float2 (&x)[8]) const {
#pragma unroll
        for (int k = 0; k < NP; ++k) {
            const uint4 u = *place(slot, k);
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int j = 0; j < F; ++j) {
                if constexpr (sizeof(T) == 2)
                    x[k * F + j] = make_float2(__uint_as_float(w[j] << 16), __uint_as_float(w[j] & 0xffff0000u));
                else
                    x[k * F + j] = make_float2(__uint_as_float(w[2 * j]), __uint_as_float(w[2 * j + 1]));
            }
        }
    }
};
template <typename T, bool VEC>
__device__ __forceinline__ void store_chunk(T* p, const float2* x) {
    constexpr int E = Chunks<T>::E;
    __align__(16) T t[E];
#pragma unroll
    for (int j = 0; j < E / 2; ++j) {
        if constexpr (sizeof(T) == 2) {
            reinterpret_cast<uint32_t*>(t)[j] = pack_bf16(x[j].x, x[j].y);
        } else {
            t[2 * j] = x[j].x;
            t[2 * j + 1] = x[j].y;
        }
    }
    if constexpr (VEC) {
        *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(t);
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i) p[i] = t[i];
    }
}

// Rows of a token, one after the other: queries of a layer, its keys, the next layer's.  Those of a side and layer lie one stride apart.
struct RowWalk {
    const RotateArgs& r;
    int heads, layer, h;
    long long at, step;  // element offset of the row, within its side
    __device__ RowWalk(const RotateArgs& r, int row) : r(r), heads(r.side[0].heads + r.side[1].heads), layer(row / heads), h(row - layer * heads) {}
    __device__ __forceinline__ bool second() const { return h >= r.side[0].heads; }
    // OUT: of the outputs; c, i: the token
    template <bool OUT>
    __device__ __forceinline__ void place(int c, int i) {
        const RotateSide& s = r.side[second()];
        const long long* d = OUT ? s.o : s.s;
        at = c * d[0] + layer * d[1] + (second() ? h - r.side[0].heads : h) * d[2] + i * d[3];
        step = d[2];
    }
    template <bool OUT>
    __device__ __forceinline__ void next(int c, int i) {
        ++h;
        if (h == heads || h == r.side[0].heads) {
            if (h == heads) h = 0, ++layer;
            place<OUT>(c, i);
        } else {
            at += step;
        }
    }
};

// HD / 16 lanes take a job: some rows of one token, whose angles they compute once.  A lane has 16 elements of each row, with both of a pair, so that
// a row takes no exchange but its sum of squares.
// Bound by HBM and, in bf16, nearly by instructions (67% of the issue slots; fp32 two at a time; an angle's cosine and sine, 45 of them, once for 16
// rows): 2048 tokens of 16 layers, 40 heads of 64 in 57 us, 336 MB at 5.8 TB/s, of 128 in 104 (6.4); in fp32 104 and 199 (6.5, 6.7; a copy
// reaches 6.8).  The ring is what keeps enough bytes under way: a row at a time took 79 us, the next row's chunks in registers 90 (104 of
// them, 14 warps an SM); a ring of 6 rows or jobs of 32 the same to 3% more.  Chunks of neighbouring lanes lie beside one another, so that an
// instruction takes whole sectors: with two chunks of a lane beside one another fp32 took 139, neighbouring pairs 74 for 59.  Five
// CTAs an SM (102 registers) for four: 59 for 63.  One token is bound by its launch and three dependent loads (2.5 us in a graph; with a branch
// for each pair that may not turn 3.0).
template <typename T, int HD, bool VEC>
__global__ void __launch_bounds__(NR_THREADS, 5) norm_rotate_kernel(const __grid_constant__ NormRotateArgs a) {
    constexpr int LANES = HD / 16, E = Chunks<T>::E, NP = Chunks<T>::NP, H = Chunks<T>::H, F = Chunks<T>::F;
    extern __shared__ __align__(16) uint8_t nr_smem[];
    const Ring<T, VEC> ring(nr_smem);
    const RotateArgs& r = a.r;
    pdl_wait();
    const long long job = ((long long)blockIdx.x * NR_THREADS + threadIdx.x) / LANES;
    const int l = threadIdx.x % LANES;
    const long long tokens = (long long)r.n_ctx * r.n_tok;
    const bool live = job < a.jobs;
    const long long part = live ? job / tokens : 0, ct = live ? job - part * tokens : 0;
    const int c = (int)(ct / r.n_tok), i = (int)(ct - (long long)c * r.n_tok);
    // The chunks: those of neighbours in order; of halves H of each half, first those that turn, then those of the halves of what does not
    int d[NP];
#pragma unroll
    for (int k = 0; k < NP; ++k) {
        const int t = (r.neighbours ? k : k % H) * LANES + l, over = t * E - r.rot / 2;  // of the first half
        if (r.neighbours)
            d[k] = t * E;
        else if (over < 0)
            d[k] = t * E + k / H * (r.rot / 2);
        else
            d[k] = r.rot + over + k / H * ((HD - r.rot) / 2);
    }
    const int row0 = (int)part * a.chunk, rows = live ? min(a.chunk, a.rows - row0) : 0;
    RowWalk in(r, row0), out(r, row0);
    in.place<false>(c, i);
    out.place<true>(c, i);
    auto copy = [&](int n) {
        if (n < rows) {
            const T* x = static_cast<const T*>(r.side[in.second()].x) + in.at;
            ring.copy(n % NR_DEPTH, x, d);
            in.next<false>(c, i);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int n = 0; n < NR_DEPTH - 1; ++n) copy(n);
    float2 co[4], si[4];  // of this lane's pairs 2 e and 2 e + 1
    unsigned turns = 0;   // which of them turn
    {
        unsigned p = (unsigned)((r.first ? r.first[c] : 0) + i);
        if (r.period) p %= (unsigned)r.period;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int pair = r.neighbours ? (e / F * LANES + l) * F + e % F : (e / E * LANES + l) * E + e % E;
            const bool on = pair < r.rot / 2;  // (below 64 in any case, what the table has)
            float x, y;
            cos_sin(on ? r.turns[pair] * p : 0, x, y);
            turns |= on << e;
            (e & 1 ? co[e / 2].y : co[e / 2].x) = x;
            (e & 1 ? si[e / 2].y : si[e / 2].x) = y;
        }
    }
    float2 w[8];
    const float* loaded = nullptr;
#pragma unroll 1
    for (int n = 0; n < a.chunk; ++n) {
        const bool on = n < rows;
        if (!__any_sync(0xffffffffu, on)) break;
        copy(n + NR_DEPTH - 1);
        const RotateSide& s = r.side[out.second()];
        const bool scaled = on && s.w;
        const float* weight = s.w + (size_t)out.layer * HD;
        if (scaled && weight != loaded) {  // a layer's, of a side
            loaded = weight;
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = make_float2(weight[d[e / F] + 2 * (e % F)], weight[d[e / F] + 2 * (e % F) + 1]);
        }
        asm volatile("cp.async.wait_group %0;" ::"n"(NR_DEPTH - 1) : "memory");
        float2 x[8];
        ring.read(n % NR_DEPTH, x);
        if (__any_sync(0xffffffffu, scaled)) {
            auto squares = [&]() {
                float2 s = make_float2(0.f, 0.f);
#pragma unroll
                for (int e = 0; e < 8; ++e) s = fma2(x[e], x[e], s);
                float ss = s.x + s.y;
#pragma unroll
                for (int o = 1; o < LANES; o <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
                return ss;
            };
            float mean = squares() / HD + r.eps;
            const bool out_of_range = scaled && !(mean > 1e-30f && mean < 1e37f);
            if (__any_sync(0xffffffffu, out_of_range)) {  // squares that 32 bits do not hold: of the row scaled by a power of two
                if (out_of_range) {
                    const float scale = mean <= 1e-30f ? 0x1p80f : 0x1p-70f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = mul2(x[e], make_float2(scale, scale));
                    mean = r.eps * scale * scale;
                } else {
                    mean = r.eps;
                }
                mean += squares() / HD;
            }
            if (scaled) {
                const float inv = rsqrtf(mean);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = mul2(x[e], mul2(w[e], make_float2(inv, inv)));
            }
        }
        auto rotate = [&](auto every) {  // what does not turn is left alone: 0 times an infinity is not 0
            constexpr bool EVERY = decltype(every)::value;
            if (r.neighbours) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float co1 = e & 1 ? co[e / 2].y : co[e / 2].x, si1 = e & 1 ? si[e / 2].y : si[e / 2].x;
                    if (EVERY || (turns >> e & 1)) x[e] = make_float2(x[e].x * co1 - x[e].y * si1, x[e].y * co1 + x[e].x * si1);
                }
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 p = x[e], q = x[4 + e];
                    if (EVERY || (turns >> (2 * e) & 1)) {
                        x[e] = fma2(p, co[e], mul2(q, make_float2(-si[e].x, -si[e].y)));
                        x[4 + e] = fma2(q, co[e], mul2(p, si[e]));
                    }
                }
            }
        };
        r.rot == HD ? rotate(std::true_type()) : rotate(std::false_type());
        if (on) {
            T* to = static_cast<T*>(s.out) + out.at;
#pragma unroll
            for (int k = 0; k < NP; ++k) store_chunk<T, VEC>(to + d[k], x + k * F);
            out.next<true>(c, i);
        }
    }
}

template <typename T, int HD, bool VEC>
cudaError_t launch(const NormRotateArgs& a, cudaStream_t st) {
    const long long threads = a.jobs * (HD / 16);
    return launch_kernel(norm_rotate_kernel<T, HD, VEC>, dim3((unsigned)((threads + NR_THREADS - 1) / NR_THREADS)), dim3(NR_THREADS), Ring<T, VEC>::BYTES, st,
                         true, 1, a);
}
template <typename T, int HD>
cudaError_t launch(const NormRotateArgs& a, bool vec, cudaStream_t st) {
    return vec ? launch<T, HD, true>(a, st) : launch<T, HD, false>(a, st);
}

}  // namespace

cudaError_t launch_norm_rotate(const DevState& s, const RotateArgs& r, cudaStream_t st) {
    NormRotateArgs a{r, r.L * (r.side[0].heads + r.side[1].heads), 1, 0};
    const long long tokens = (long long)r.n_ctx * r.n_tok;
    while (a.chunk < NR_CHUNK && 2 * a.chunk <= a.rows && tokens * a.rows / (2 * a.chunk) * (s.hd / 16) >= NR_FILL) a.chunk *= 2;
    a.jobs = tokens * ((a.rows + a.chunk - 1) / a.chunk);
    if (a.jobs * (s.hd / 16) > (long long)INT_MAX * NR_THREADS) return cudaErrorInvalidValue;  // (more rows than any memory has)
    uintptr_t all = 0;
    for (const RotateSide& x : r.side) {
        if (!x.heads) continue;
        all |= (uintptr_t)x.x | (uintptr_t)x.out;
        for (int i = 0; i < 4; ++i) all |= (uintptr_t)((x.s[i] | x.o[i]) * (s.dtype == 0 ? 4 : 2));
    }
    const bool vec = (all & 15u) == 0;
    if (s.dtype == 0) return s.hd == 64 ? launch<float, 64>(a, vec, st) : launch<float, 128>(a, vec, st);
    return s.hd == 64 ? launch<bf16, 64>(a, vec, st) : launch<bf16, 128>(a, vec, st);
}

}  // namespace mone
