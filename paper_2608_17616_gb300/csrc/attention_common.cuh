// What the consumer attention's forms (attention.cu) and the windowed prefill form (attention_window.cu) share.
#pragma once

#include "mone_common.cuh"

namespace mone {

struct AttnArgs {
    const void* Q;          // [C][n_q][Lq][hd]
    const void *K, *V;      // caches, element strides s0 (context), s1 (layer), s2 (head), s3 (position)
    void* out;              // [C][n_q][Lq][hd]
    long long s0, s1, s2, s3;
    int L, n_q, n_kv, group, Lq, n_mem, rows;  // rows: query tokens per CTA (group * rows <= ATT_ITEMS)
    float scale;            // 1 / sqrt(hd)
    int tile_tok, per_block;  // decode form: tokens of a block, 16-row tiles that cut it
    int group_inv;            // decode form: 65536 / group + 1
    int n_sink, window;     // windowed: a token at position t sees j <= t with j < n_sink or j > t - window
    int vec;                // caches 16-byte aligned (base and every stride): stage with 16-byte loads
    int* status;            // device status word (bounded waits of the prefill form)
};

// The chunks of STEP positions that hold the keys of the tokens at positions t0 .. t1: those of the first
// positions, then those from the first token's window on.  Every position is in one chunk at most.
struct WinRange {
    int ns, lo, n;  // chunks of the first positions; first position after them; chunks in all
    __device__ WinRange(const AttnArgs& a, int t0, int t1, int step) {
        ns = (min(a.n_sink, t1 + 1) + step - 1) / step;
        lo = max(ns * step, t0 - a.window + 1);
        n = ns + (lo <= t1 ? (t1 - lo) / step + 1 : 0);
    }
    __device__ int at(int j, int step) const { return j < ns ? j * step : lo + (j - ns) * step; }
};

// Output dimensions d0, d0 + STEP, .. of one row over the keys it sees and no others, by one thread.  A tile's
// products take a key's value row times a probability of 0 for the rows that do not see it, which is NaN where the
// value is not finite; a row of the windowed attention with such a result is computed again here.  One pass with
// a running maximum; slow, and reached by non-finite inputs only.
template <typename T, int HD, int N, int STEP>
__device__ __noinline__ void row_again(const T* q, const T* K, const T* V, long long s3, int vis, const AttnArgs& a, int d0, float* o) {
    float m = -INFINITY, l = 0.f;
    for (int d = 0; d < N; ++d) o[d] = 0.f;
    for (int j = min(a.n_sink, vis) > 0 ? 0 : max(0, vis - a.window); j < vis; ++j) {
        if (j >= a.n_sink && j < vis - a.window) j = vis - a.window;
        if (j >= vis) break;
        float z = 0.f;
        for (int d = 0; d < HD; ++d) z = fmaf(to_f<T>(q[d]), to_f<T>(K[(long long)j * s3 + d]), z);
        z *= a.scale;
        if (z == -INFINITY) continue;
        const float mn = fmaxf(m, z), corr = __expf(m - mn), p = __expf(z - mn);
        m = mn;
        l = fmaf(l, corr, p);
        for (int d = 0; d < N; ++d) o[d] = fmaf(o[d], corr, p * to_f<T>(V[(long long)j * s3 + d0 + STEP * d]));
    }
    const float inv = l > 0.f ? 1.f / l : l;
    for (int d = 0; d < N; ++d) o[d] *= inv;
}

// 2^x on the special-function unit (PTX ex2.approx), whose error is far below the bf16
// rounding of the probabilities it feeds (the parity tests bound the result at 1e-2).
__device__ __forceinline__ float at_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// The windowed prefill form (bf16, 16-byte-aligned rows), in attention_window.cu.  cudaErrorNotSupported: strides past a tensor map's range.
cudaError_t launch_window_prefill(const AttnArgs& a, int hd, int n_ctx, int C, int sms, cudaStream_t st);
// Its CUDA-core form: fp32 (dtype 0), and bf16 rows of any alignment.
cudaError_t launch_window_cores(AttnArgs a, int dtype, int hd, int C, cudaStream_t st);

}  // namespace mone
