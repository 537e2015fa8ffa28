// Queries and keys normalised by head and rotated by position, in one pass (mone_norm_rotate).
#include <algorithm>
#include <climits>

#include "mone_common.cuh"

namespace mone {

namespace {

constexpr int NR_THREADS = 128;

struct NormRotateArgs {
    RotateArgs r;
    int rows, chunk;  // rows of a token (every layer, every head of both sides); of them, those of a job
    long long jobs;
};

// cos and sin of an angle of `turn` 2^-64ths of a whole turn.  The nearest quarter turn is taken off exactly, so that the angle that is left,
// an eighth of a turn at most, is rounded to 24 bits of itself.
__device__ __forceinline__ void cos_sin(unsigned long long turn, float& c, float& s) {
    const uint32_t hi = (uint32_t)(turn >> 32);
    const uint32_t quarter = (hi + 0x20000000u) >> 30;
    const int32_t rest = (int32_t)(hi - (quarter << 30));
    float x, y;
    sincospif((float)rest * 0x1p-31f, &y, &x);
    c = quarter & 1 ? -y : x;
    s = quarter & 1 ? x : y;
    if (quarter & 2) {
        c = -c;
        s = -s;
    }
}

// 8 neighbours
template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* p, float* x) {
    if constexpr (VEC) {
        constexpr int PER = 16 / sizeof(T);
        uint4 u[8 / PER];
#pragma unroll
        for (int i = 0; i < 8 / PER; ++i) u[i] = reinterpret_cast<const uint4*>(p)[i];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = to_f<T>(reinterpret_cast<const T*>(&u[i / PER])[i % PER]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = to_f<T>(p[i]);
    }
}
template <typename T, bool VEC>
__device__ __forceinline__ void store8(T* p, const float* x) {
    if constexpr (VEC) {
        __align__(16) T t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = from_f<T>(x[i]);
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(p)[i] = reinterpret_cast<const uint4*>(t)[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = from_f<T>(x[i]);
    }
}

// HD / 16 lanes take a job: some rows of one token, whose angles they compute once.  A lane has two pieces of eight elements of each row, for
// halves those that are paired, so that a row takes no exchange but its sum of squares.
template <typename T, int HD, bool VEC>
__global__ void __launch_bounds__(NR_THREADS) norm_rotate_kernel(const __grid_constant__ NormRotateArgs a) {
    constexpr int LANES = HD / 16;
    const RotateArgs& r = a.r;
    pdl_wait();
    const long long job = ((long long)blockIdx.x * NR_THREADS + threadIdx.x) / LANES;
    const int l = threadIdx.x % LANES;
    const bool live = job < a.jobs;
    const long long tokens = (long long)r.n_ctx * r.n_tok;
    const long long part = live ? job / tokens : 0, ct = live ? job - part * tokens : 0;
    const int c = (int)(ct / r.n_tok), i = (int)(ct - (long long)c * r.n_tok);
    const int n_rot = r.rot / 16;
    const bool turns = l < n_rot;
    const int d0 = 8 * (turns && !r.neighbours ? l : 2 * l), d1 = turns && !r.neighbours ? d0 + r.rot / 2 : d0 + 8;
    float co[8], si[8];
    {
        unsigned p = (unsigned)((r.first ? r.first[c] : 0) + i);
        if (r.period) p %= (unsigned)r.period;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            co[e] = 1.f;
            si[e] = 0.f;
            if (turns) cos_sin(r.turns[8 * l + e] * p, co[e], si[e]);
        }
    }
    const int heads = r.side[0].heads + r.side[1].heads;
    const int row0 = (int)part * a.chunk, row1 = live ? min(row0 + a.chunk, a.rows) : row0;
    for (int n = 0; n < a.chunk; ++n) {
        const int row = min(row0 + n, a.rows - 1), layer = row / heads, h = row - layer * heads;
        const bool second = h >= r.side[0].heads, on = row0 + n < row1;
        const RotateSide& s = r.side[second];
        const int head = second ? h - r.side[0].heads : h;
        float x[16], ss;
        const T* from = static_cast<const T*>(s.x) + c * s.s[0] + layer * s.s[1] + head * s.s[2] + i * s.s[3];
        if (on) {
            load8<T, VEC>(from + d0, x);
            load8<T, VEC>(from + d1, x + 8);
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] = 0.f;
        }
        auto squares = [&]() {
            ss = 0.f;
#pragma unroll
            for (int e = 0; e < 16; ++e) ss = fmaf(x[e], x[e], ss);
#pragma unroll
            for (int o = 1; o < LANES; o <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        };
        squares();
        float mean = ss / HD + r.eps;
        const bool out_of_range = s.w && !(mean > 1e-30f && mean < 1e37f);
        if (__any_sync(0xffffffffu, out_of_range)) {  // squares that 32 bits do not hold: of the row scaled by a power of two
            if (out_of_range) {
                const float scale = mean <= 1e-30f ? 0x1p80f : 0x1p-70f;
#pragma unroll
                for (int e = 0; e < 16; ++e) x[e] *= scale;
                mean = r.eps * scale * scale;
            } else {
                mean = r.eps;
            }
            squares();
            mean += ss / HD;
        }
        if (s.w) {
            const float inv = rsqrtf(mean);
            const float* w = s.w + (size_t)layer * HD;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[e] *= inv * w[d0 + e];
                x[8 + e] *= inv * w[d1 + e];
            }
        }
        if (turns) {
            if (r.neighbours) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float p = x[2 * e], q = x[2 * e + 1];
                    x[2 * e] = p * co[e] - q * si[e];
                    x[2 * e + 1] = q * co[e] + p * si[e];
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float p = x[e], q = x[8 + e];
                    x[e] = p * co[e] - q * si[e];
                    x[8 + e] = q * co[e] + p * si[e];
                }
            }
        }
        if (on) {
            T* to = static_cast<T*>(s.out) + c * s.o[0] + layer * s.o[1] + head * s.o[2] + i * s.o[3];
            store8<T, VEC>(to + d0, x);
            store8<T, VEC>(to + d1, x + 8);
        }
    }
}

template <typename T, int HD, bool VEC>
cudaError_t launch(const NormRotateArgs& a, cudaStream_t st) {
    const long long threads = a.jobs * (HD / 16);
    return launch_kernel(norm_rotate_kernel<T, HD, VEC>, dim3((unsigned)((threads + NR_THREADS - 1) / NR_THREADS)), dim3(NR_THREADS), 0, st, true, 1, a);
}
template <typename T, int HD>
cudaError_t launch(const NormRotateArgs& a, bool vec, cudaStream_t st) {
    return vec ? launch<T, HD, true>(a, st) : launch<T, HD, false>(a, st);
}

}  // namespace

cudaError_t launch_norm_rotate(const DevState& s, const RotateArgs& r, cudaStream_t st) {
    NormRotateArgs a{r, r.L * (r.side[0].heads + r.side[1].heads), 1, 0};
    const long long tokens = (long long)r.n_ctx * r.n_tok;
    while (a.chunk < 8 && 2 * a.chunk <= a.rows && tokens * a.rows / (2 * a.chunk) >= 16384) a.chunk *= 2;
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
