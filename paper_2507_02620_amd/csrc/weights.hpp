// What the kernels that draw from logits share: the whole-number weights of scores, rows by pieces, sums over a wave.
#pragma once
#include "common.hpp"

#include <math.h>

#pragma clang fp contract(off)

// Operations that are rounded by themselves.  (The runtime's __fmul_rn and __fsub_rn are plain operators compiled without the pragma above: a product
// and the difference behind it became one fused step where the product had no other use, and a score on the border of a bin fell to either side.)
static __device__ __forceinline__ float mul_once(float a, float b) { return a * b; }
static __device__ __forceinline__ float sub_once(float a, float b) { return a - b; }

// E = (uint64)(exp2_spec * 2^32).  The polynomial's value p lies in [1, 2]; scaling it by 2^(n + 32), n <= 0, and truncating is a
// shift of its 24-bit significand, exact and without the conversion sequence a float -> uint64 cast takes.
static __device__ __forceinline__ uint64_t exp_weight(float z, float m) {
    const float t = mul_once(sub_once(z, m), 1.44269504088896341f);  // <= 0: m is the row's maximum
    if (!(t >= -64.0f)) return 0;
    const float n = floorf(t), f = sub_once(t, n);
    float p = 1.52527338e-5f;
    p = fmaf(p, f, 1.54035304e-4f);
    p = fmaf(p, f, 1.33335581e-3f);
    p = fmaf(p, f, 9.61812911e-3f);
    p = fmaf(p, f, 5.55041087e-2f);
    p = fmaf(p, f, 2.40226507e-1f);
    p = fmaf(p, f, 6.93147181e-1f);
    p = fmaf(p, f, 1.0f);
    const unsigned bits = __float_as_uint(p);
    const int sh = 127 - (int)(bits >> 23) - (int)n;  // 0 .. 64 places below 2^32 (p = 2 only with n <= -1)
    // (the shift in 32 bits, with the cases of no and of more than 32 places apart, makes the sums' launch 12.8 -> 14.2 us)
    return ((uint64_t)((bits & 0x7FFFFFu) | 0x800000u) << 9) >> min(sh, 63);
}

// Row maxima are kept as unsigned keys that order like the floats do (0: below every float), so that the chunks of a row can
// meet in an atomic maximum.
static __device__ __forceinline__ unsigned max_key(float m) {
    const unsigned b = __float_as_uint(m);
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
static __device__ __forceinline__ float key_max(unsigned k) { return __uint_as_float((k & 0x80000000u) ? (k & 0x7FFFFFFFu) : ~k); }

// Visits n pieces of E floats with all threads of the group, adjacent threads on adjacent pieces, U loads in flight per thread.  fn(x, live, index).
// CLAMP: what a thread has left behind its full rounds goes out together too and repeats the last piece (live is false for repeats) instead of
// one load at a time: shorter where a round is most of the work, longer where it is little of it.
template <int U, bool CLAMP, int E, typename F>
static __device__ __forceinline__ void for_pieces(const float* __restrict__ p, int n, int t, int nt, F&& fn) {
    auto load = [&](int i, float (&x)[E]) __attribute__((always_inline)) {
        if constexpr (E == 4) {
            const f32x4 q = *(const f32x4*)(p + (size_t)i * 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = q[e];
        } else {
            x[0] = p[i];
        }
    };
    int i = t;
    for (; i + (U - 1) * nt < n; i += U * nt) {
        float x[U][E];
#pragma unroll
        for (int k = 0; k < U; ++k) load(i + k * nt, x[k]);
#pragma unroll
        for (int k = 0; k < U; ++k)
#pragma unroll
            for (int e = 0; e < E; ++e) fn(x[k][e], true, (i + k * nt) * E + e);
    }
    if constexpr (CLAMP) {
        if (i < n) {
            float x[U][E];
#pragma unroll
            for (int k = 0; k < U; ++k) load(min(i + k * nt, n - 1), x[k]);
#pragma unroll
            for (int k = 0; k < U; ++k)
#pragma unroll
                for (int e = 0; e < E; ++e) fn(x[k][e], i + k * nt < n, (i + k * nt) * E + e);
        }
    } else {
        for (; i < n; i += nt) {
            float x[E];
            load(i, x);
#pragma unroll
            for (int e = 0; e < E; ++e) fn(x[e], true, i * E + e);
        }
    }
}

// The elements [lo, hi) of a row: by 16 bytes where the row allows it (lo a multiple of 4), the rest by elements.
template <int U, bool CLAMP, typename F>
static __device__ __forceinline__ void for_row(const float* __restrict__ p, int lo, int hi, int t, int nt, bool vec, F&& fn) {
    int v = lo;
    if (vec) {
        for_pieces<U, CLAMP, 4>(p + lo, (hi - lo) >> 2, t, nt, [&](float x, bool live, int i) { fn(x, live, lo + i); });
        v = lo + ((hi - lo) & ~3);
    }
    for_pieces<U, CLAMP, 1>(p + v, hi - v, t, nt, [&](float x, bool live, int i) { fn(x, live, v + i); });
}

static __device__ __forceinline__ uint64_t wave_sum_u64(uint64_t v) {
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, FS_WAVE);
    return v;
}

// Running sum of v over the lanes, this lane's included.
static __device__ __forceinline__ uint64_t wave_scan_u64(uint64_t v) {
    const int lane = threadIdx.x & 63;
    for (int o = 1; o < 64; o <<= 1) {
        const uint64_t below = __shfl_up(v, o, FS_WAVE);
        if (lane >= o) v += below;
    }
    return v;
}
