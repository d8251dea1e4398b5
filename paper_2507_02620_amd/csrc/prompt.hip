// Causal attention over whole prompts packed behind one another, grouped heads.
#include "paged.hpp"
#include "rows_attn.hpp"

#include <algorithm>
#include <vector>

namespace {

// What a workgroup does: a block of rows of a sequence, in one head.
struct Unit {
    int start, len, block, qh;
};

// Unit `id` of a launch.  Units come in levels of `width` block indices, the highest first (the blocks with the most slots before them start
// first), in a level by sequence, the longest first, then by head: consecutive ids, which go to the XCDs in turn, differ in the KV head, so that with 8
// heads or a divisor of 8 each XCD's L2 holds its own heads (4096 tokens, 16/8 heads of 64: 62.3 -> 59.7 us; 20 prompts of 100 tokens, 28/4 heads: 23.1 -> 21.7).  Where all units run at once, two to a compute unit, the second half of
// the ids takes the lighter units in ascending order: the lightest beside the heaviest (2048 tokens, 32 heads:
// 53.8 -> 50.2 us).
static __device__ __forceinline__ bool unit_of(const PromptArgs& a, int id, Unit& u) {
    if (a.units <= 2 * a.cus && id >= a.cus) id = a.cus + a.units - 1 - id;
    const int f = id / a.Hq, y = id - f * a.Hq;
    u.qh = y % a.Hkv * a.G + y / a.Hkv;
    int d = 0;  // the last level that begins at or before f
    const int lane = threadIdx.x & 63;
    for (int i = 0; i < a.levels; i += 64) d += __popcll(__ballot(i + lane < a.levels && a.first[min(i + lane, PROMPT_MAX_SEQ - 1)] <= f));
    d = __builtin_amdgcn_readfirstlane(d - 1);
    const int r = f - a.first[d], sq = r / a.width;
    u.block = (a.levels - 1 - d) * a.width + a.width - 1 - r % a.width;
    u.start = a.start[sq];
    u.len = a.len[sq];
    return u.block * a.rows < u.len;
}

// Every `step`-th half of 32 slots from the first-th on for 16 rows of a sequence, by one wave, keys and values from memory (L2).
template <typename T, int HD>
static __device__ __forceinline__ void rows16(RowTiles<T, HD, 1>& rt, const PromptArgs& a, int start, int len, int r0, int qh, int first, int step, T* vt,
                                              int lane) {
    const int r16 = lane & 15, g = lane >> 4, kvh = qh / a.G;
    rt.init();
    const bool ok = r0 + r16 < len;
    rt.load_q(0, (const T*)a.q + (long long)(start + (ok ? r0 + r16 : r0)) * a.q_tok + (long long)qh * a.q_head, ok, g);
    const T* kb = (const T*)a.k + (long long)start * a.k_tok + (long long)kvh * a.k_head;
    const T* vb = (const T*)a.v + (long long)start * a.v_tok + (long long)kvh * a.v_head;
    const int end = min(len, r0 + 16);  // slots the last row sees
    for (int s0 = first * 32; s0 < end; s0 += step * 32) {
        const int n = r0 + r16 + 1 - s0;
        unsigned vis[1] = {!ok || n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1};
        const T *kp = kb + (long long)s0 * a.k_tok, *vp = vb + (long long)s0 * a.v_tok;
        if (s0 + 32 <= r0 + 1) rt.template half<false>(kp, vp, a.k_tok, a.v_tok, 31, vis, a.scale_log2, vt, lane);
        else rt.template half<true>(kp, vp, a.k_tok, a.v_tok, min(31, len - 1 - s0), vis, a.scale_log2, vt, lane);
    }
}

// f32: a workgroup per 16 rows of a head, whose waves take every fourth half of 32 slots and meet in LDS.  Bound by the f32 matrix
// instructions (32 cycles for 2048 products) and, for short prompts, by one wave's chain of halves, which the split over waves shortens
// (1000 tokens, 4 heads: 73 us with a wave per 16 rows -> 19.5).
template <typename T, int HD>
__global__ void __launch_bounds__(256) prompt_rows_kernel(const PromptArgs a) {
    using RT = RowTiles<T, HD, 1>;
    constexpr int RROW = HD + 4, STAGE = 4 * RT::STAGE * (int)sizeof(T), RED = 4 * 16 * (RROW + 2) * 4;
    __shared__ __align__(16) unsigned char lds[STAGE > RED ? STAGE : RED];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), r16 = lane & 15, g = lane >> 4;
    Unit un;
    if (!unit_of(a, blockIdx.x, un)) return;
    const int r0 = un.block * 16;
    RT rt;
    rows16<T, HD>(rt, a, un.start, un.len, r0, un.qh, w, 4, (T*)lds + w * RT::STAGE, lane);
    const float l = rt.row_sum(0);
    __syncthreads();
    float *ro = (float*)lds, *rml = ro + 4 * 16 * RROW;
#pragma unroll
    for (int n = 0; n < HD / 16; ++n) *(f32x4*)(ro + (w * 16 + r16) * RROW + n * 16 + g * 4) = rt.acc[0][n];
    if (g == 0) *(float2*)(rml + (w * 16 + r16) * 2) = make_float2(rt.m[0], l);
    __syncthreads();
    const int row = tid >> 4;
    if (r0 + row >= un.len) return;
    float2 ml[4];
    float mm = FS_NEG_INF;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        ml[k] = *(const float2*)(rml + (k * 16 + row) * 2);
        mm = fmaxf(mm, ml[k].x);
    }
    const float ms = mm == FS_NEG_INF ? 0.f : mm;
    float den = 0.f, wt[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        wt[k] = __builtin_amdgcn_exp2f(ml[k].x - ms);
        den += wt[k] * ml[k].y;
    }
    const float inv = 1.0f / den;
    T* op = (T*)a.o + (long long)(un.start + r0 + row) * a.o_tok + (long long)un.qh * a.o_head + (tid & 15) * 4;
#pragma unroll
    for (int c = 0; c < HD / 64; ++c) {
        f32x4 o{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < 4; ++k) o += *(const f32x4*)(ro + (k * 16 + row) * RROW + (tid & 15) * 4 + c * 64) * wt[k];
        *(typename RT::E::out4_t*)(op + c * 64) = RT::E::pack4(o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
    }
}

// bf16: a workgroup per 128 rows of a head, a wave per 32.
//
// S^T = K . Q^T and O^T += V^T . P^T by 32x32x16 products: lane l holds values of query row l % 32 only (two lanes to a row), so the
// softmax state is per lane and P never leaves registers: S^T has slot 8 (v / 4) + 4 (l / 32) + v % 4 in register v, which is
// the order in which the V^T operand is read with the transposing LDS load.  K/V tiles of 64 slots go from memory straight into LDS, two
// buffers, one barrier per tile, rows swizzled against bank conflicts.
// Two workgroups share a compute unit, or two groups of four waves in one workgroup take alternate tiles (GROUPS = 2) and join
// their sums in LDS at the end: one wave's exponentials run behind the other's matrix products.
//
// The running maximum is only raised where a score exceeds it by more than 2^8 in the exponential (any common factor of numerator and
// denominator is as good; 8 bits of headroom cost no precision in floating point), so most tiles rescale nothing.
// A masked slot's V row is multiplied by zero, which a value that is not finite would survive: a wave that ends with any such sum does
// its rows again slot by slot.
typedef float f32x16 __attribute__((ext_vector_type(16)));

// The larger of a lane's value and that of the lane 32 away.
static __device__ __forceinline__ float half_max(float x) {
    typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
    const u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Where a row's 16-byte chunks lie in LDS: chunk c at place c ^ swizzle(row).  The 64 banks hold one row of 128 columns or two of 64.  A K read takes one
// chunk of 16 rows: all 16 places differ (64 columns: 8 of them for the rows of either half of the banks).  A transposing V read takes four
// neighbouring chunks of four rows from a multiple of 4 on: the rows' lowest bits choose the group of four.  (c ^ row, which suits the K read
// as well, sends all four rows to one group: 60 % of LDS cycles were conflicts.)
template <int HD>
static __device__ __forceinline__ unsigned swizzle(unsigned r) {
    return HD == 128 ? (r & 3) << 2 | (r >> 2 & 3) : (r >> 1 & 1) << 2 | (r >> 2 & 1) << 1 | (r >> 3 & 1);
}

template <int HD, int GROUPS>
__global__ void __launch_bounds__(512) prompt_tiles_kernel(const PromptArgs a) {
    using E = Elem<bf16_t>;
    constexpr int BS = 64, ROWB = HD * 2, CHUNKS = ROWB / 16, NKT = HD / 16, NHT = HD / 32, TILE = BS * ROWB;
    constexpr int RPL = 1024 / ROWB, LPW = BS / RPL / 4;  // rows per direct-to-LDS load of a wave; such loads per wave and tile (K, and V)
    constexpr float HEADROOM = 8.f;
    __shared__ __align__(1024) unsigned char tb0[GROUPS * 2 * TILE];
    __shared__ __align__(1024) unsigned char tb1[GROUPS * 2 * TILE];
    constexpr int STAGE = RowTiles<bf16_t, HD, 1>::STAGE;
    static_assert(2 * STAGE * 2 <= 2 * TILE, "two waves' stages fit one buffer");

    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6 & 3), c32 = lane & 31, h = lane >> 5;
    const int grp = GROUPS > 1 ? __builtin_amdgcn_readfirstlane(tid >> 8) : 0;
    Unit un;
    if (!unit_of(a, blockIdx.x, un)) return;
    const int start = un.start, len = un.len, qh = un.qh, kvh = qh / a.G;
    const int blk0 = un.block * 128, r0 = blk0 + w * 32, row = r0 + c32;
    const bool ok = row < len;
    const int tiles = (min(len, blk0 + 128) + BS - 1) / BS;  // slots the block's last row sees

    bf16x8 qf[NKT];
    {
        const bf16_t* qp = (const bf16_t*)a.q + (long long)(start + (ok ? row : 0)) * a.q_tok + (long long)qh * a.q_head + h * 8;
#pragma unroll
        for (int kt = 0; kt < NKT; ++kt) qf[kt] = ok ? *(const bf16x8*)(qp + kt * 16) : E::zero();
    }
    f32x16 acc[NHT];
#pragma unroll
    for (int n = 0; n < NHT; ++n)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[n][v] = 0.f;
    float m = FS_NEG_INF, ms = 0.f, l = 0.f;  // ms: what is subtracted, m where that is finite

    const unsigned char* kb = (const unsigned char*)((const bf16_t*)a.k + (long long)start * a.k_tok + (long long)kvh * a.k_head);
    const unsigned char* vb = (const unsigned char*)((const bf16_t*)a.v + (long long)start * a.v_tok + (long long)kvh * a.v_head);
    // Load i of a wave brings rows RPL (LPW w + i) + lane / CHUNKS, whose swizzle differs from the first load's in i alone; only behind the last
    // whole tile are rows clamped (they re-read the sequence's last one and are masked).
    const unsigned kst = (unsigned)a.k_tok * 2, vst = (unsigned)a.v_tok * 2;
    const unsigned row_w = RPL * LPW * w + lane / CHUNKS, koff = row_w * kst, voff = row_w * vst;
    const unsigned col0 = ((lane % CHUNKS) ^ swizzle<HD>(row_w)) * 16;
    auto issue = [&](int t, unsigned char* buf) __attribute__((always_inline)) {
        const unsigned char *kt = kb + (long long)t * BS * a.k_tok * 2, *vt = vb + (long long)t * BS * a.v_tok * 2;
        unsigned char* to = buf + RPL * LPW * w * ROWB;
        if ((t + 1) * BS <= len) {
#pragma unroll
            for (int i = 0; i < LPW; ++i)
                __builtin_amdgcn_global_load_lds(FS_GLB_PTR(kt + (unsigned long long)i * RPL * kst + (koff + (col0 ^ (i * 16)))), FS_LDS_PTR(to + RPL * i * ROWB), 16, 0, 0);
#pragma unroll
            for (int i = 0; i < LPW; ++i)
                __builtin_amdgcn_global_load_lds(FS_GLB_PTR(vt + (unsigned long long)i * RPL * vst + (voff + (col0 ^ (i * 16)))), FS_LDS_PTR(to + TILE + RPL * i * ROWB), 16, 0, 0);
            return;
        }
        const unsigned last = len - 1 - t * BS;
#pragma unroll
        for (int i = 0; i < LPW; ++i) {
            const unsigned r = min(row_w + RPL * i, last), c = col0 ^ (i * 16);
            __builtin_amdgcn_global_load_lds(FS_GLB_PTR(kt + (r * kst + c)), FS_LDS_PTR(to + RPL * i * ROWB), 16, 0, 0);
            __builtin_amdgcn_global_load_lds(FS_GLB_PTR(vt + (r * vst + c)), FS_LDS_PTR(to + TILE + RPL * i * ROWB), 16, 0, 0);
        }
    };
    unsigned kread[NKT], vread[NHT][2];
#pragma unroll
    for (int kt = 0; kt < NKT; ++kt) kread[kt] = (unsigned)(c32 * ROWB + (((kt * 2 + h) ^ swizzle<HD>(c32)) * 16));
    {
        const int i = lane & 15, side = (lane >> 4) & 1;
#pragma unroll
        for (int n = 0; n < NHT; ++n)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int r = 8 * u + 4 * h + (i >> 2);
                vread[n][u] = (unsigned)(TILE + r * ROWB + (((n * 4 + side * 2 + ((i & 3) >> 1)) ^ swizzle<HD>(r)) * 16) + (i & 1) * 8);
            }
    }

    auto process = [&](int t, const unsigned char* buf) __attribute__((always_inline)) {
        const int s0 = t * BS;
        if (s0 > r0 + 31 || r0 >= len) return;  // wave-uniform: behind the wave's last row, or it has none
        // The order of reads, products and exponentials is pinned (sched_barrier): a group of fragments is read while the group before
        // it is multiplied, and two exponentials stand behind every product of the second half.  Left to itself the compiler waited for
        // each pair of fragments (8192 tokens, 32 heads: 583 -> 552 us).
        f32x16 st[2];
        bf16x8 kf[2][4], vf[2][NHT];
        auto load_k = [&](int grp) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) kf[grp & 1][i] = *(const bf16x8*)(buf + kread[(grp * 4 + i) % NKT] + (grp * 4 + i) / NKT * 32 * ROWB);
        };
        auto load_v = [&](int c) __attribute__((always_inline)) {
#pragma unroll
            for (int n = 0; n < NHT; ++n) {
                const s16x4 x0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(buf + vread[n][0] + c * 16 * ROWB));
                const s16x4 x1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(buf + vread[n][1] + c * 16 * ROWB));
                vf[c & 1][n] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(x0, x1, 0, 1, 2, 3, 4, 5, 6, 7));
            }
        };
        load_k(0);
#pragma unroll
        for (int grp = 0; grp < NKT / 2; ++grp) {
            if (grp + 1 < NKT / 2) load_k(grp + 1);
            else load_v(0);
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int f = grp * 4 + i, s = f / NKT, kt = f % NKT;
                if (kt == 0)
#pragma unroll
                    for (int v = 0; v < 16; ++v) st[s][v] = 0.f;
                st[s] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[grp & 1][i], qf[kt], st[s], 0, 0, 0);
            }
            __builtin_amdgcn_s_setprio(0);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (s0 + BS > r0) {  // the diagonal passes through
            const int lim = row - s0 - 4 * h;
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int v = 0; v < 16; ++v) st[s][v] = s * 32 + 8 * (v / 4) + v % 4 <= lim ? st[s][v] : FS_NEG_INF;
        }
        float mx = st[0][0];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int v = 0; v < 16; ++v) mx = fmaxf(mx, st[s][v]);
        mx = half_max(mx) * a.scale_log2;
        if (__ballot(mx > m + HEADROOM) != 0) {
            const float mnew = fmaxf(m, mx);
            ms = mnew == FS_NEG_INF ? 0.f : mnew;
            const float alpha = __builtin_amdgcn_exp2f(m - ms);
            l *= alpha;
#pragma unroll
            for (int n = 0; n < NHT; ++n)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[n][v] *= alpha;
            m = mnew;
        }
        float sum = 0.f;
        auto expo = [&](int c, int e) __attribute__((always_inline)) {  // value e of the 8 that the lane has of 16 slots
            const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(st[c / 2][(c % 2) * 8 + e], a.scale_log2, -ms));
            st[c / 2][(c % 2) * 8 + e] = x;
            sum += x;
        };
#pragma unroll
        for (int e = 0; e < 8; ++e) expo(0, e);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            if (c + 1 < 4) load_v(c + 1);
            // P rounded to the operand type, half a step of 2^-8 of a probability, of the size of the result's own rounding; the sum is of the
            // unrounded values (distance from 64 bits 2.0e-3, with P in 32 bits 1.6e-3)
            bf16x8 pf;
#pragma unroll
            for (int e = 0; e < 8; ++e) pf[e] = (bf16_t)st[c / 2][(c % 2) * 8 + e];
#pragma unroll
            for (int n = 0; n < NHT; ++n) {
                acc[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[c & 1][n], pf, acc[n], 0, 0, 0);
                if (c + 1 < 4)
#pragma unroll
                    for (int e = 0; e < 8 / NHT; ++e) expo(c + 1, n * (8 / NHT) + e);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        l += sum;
    };

    unsigned char *const mine0 = tb0 + grp * 2 * TILE, *const mine1 = tb1 + grp * 2 * TILE;
    if (grp < tiles) issue(grp, mine0);
    auto step = [&](int t, unsigned char* buf, unsigned char* other) __attribute__((always_inline)) {  // the group's tile t (there may be none)
        asm volatile("" ::: "memory");
        FS_WAIT_VM_LGKM(0, 0);
        __builtin_amdgcn_s_barrier();  // the tiles are complete for every wave; every wave is done with those before them
        asm volatile("" ::: "memory");
        if (t + GROUPS < tiles) issue(t + GROUPS, other);
        if (GROUPS == 1 || t < tiles) process(t, buf);
    };
    for (int t = 0; t < tiles; t += 2 * GROUPS) {
        step(t + grp, mine0, mine1);
        if (t + GROUPS < tiles) step(t + GROUPS + grp, mine1, mine0);
    }
    if (GROUPS > 1) {  // the second group's sums join the first's
        float* so = (float*)tb0 + w * (NHT * 16 * 64) + lane;
        float* sm = (float*)tb1 + w * 128 + lane;
        static_assert(GROUPS == 1 || 4 * NHT * 16 * 64 * 4 <= (int)sizeof(tb0), "four waves' sums fit a buffer");
        __syncthreads();
        if (grp) {
#pragma unroll
            for (int n = 0; n < NHT; ++n)
#pragma unroll
                for (int v = 0; v < 16; ++v) so[(n * 16 + v) * 64] = acc[n][v];
            sm[0] = m;
            sm[64] = l;
        }
        __syncthreads();
        if (grp) return;
        const float m2 = sm[0], mm = fmaxf(m, m2), msub = mm == FS_NEG_INF ? 0.f : mm;
        const float w1 = __builtin_amdgcn_exp2f(m - msub), w2 = __builtin_amdgcn_exp2f(m2 - msub);
        l = l * w1 + sm[64] * w2;
#pragma unroll
        for (int n = 0; n < NHT; ++n)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[n][v] = acc[n][v] * w1 + so[(n * 16 + v) * 64] * w2;
    }

    l = wave_xor_add(l, 32);
    const float inv = 1.0f / l;
    bool odd = !(fabsf(l) < __builtin_inff());
#pragma unroll
    for (int n = 0; n < NHT; ++n)
#pragma unroll
        for (int v = 0; v < 16; ++v) odd |= !(fabsf(acc[n][v]) < __builtin_inff());
    const bool again = __ballot(ok && odd) != 0;
    if (GROUPS == 1) __syncthreads();  // both buffers are free (with two groups the stages lie behind what other waves may still be reading)
    if (again) {
        bf16_t* stage = GROUPS == 1 ? (bf16_t*)(w < 2 ? tb0 : tb1) + (w & 1) * STAGE : (bf16_t*)(tb1 + 2048) + w * STAGE;
        static_assert(GROUPS == 1 || 2048 + 4 * STAGE * 2 <= (int)sizeof(tb1), "four waves' stages fit a buffer");
#pragma nounroll
        for (int i = 0; i < 2; ++i) {
            const int q0 = r0 + 16 * i, qrow = q0 + (lane & 15);
            if (q0 >= len) return;
            RowTiles<bf16_t, HD, 1> rt;
            rows16<bf16_t, HD>(rt, a, start, len, q0, qh, 0, 1, stage, lane);
            const float iv = 1.0f / rt.row_sum(0);
            bf16_t* o = (bf16_t*)a.o + (long long)(start + qrow) * a.o_tok + (long long)qh * a.o_head + (lane >> 4) * 4;
            if (qrow < len)
#pragma unroll
                for (int n = 0; n < HD / 16; ++n)
                    *(bf16x4*)(o + n * 16) = E::pack4(rt.acc[0][n][0] * iv, rt.acc[0][n][1] * iv, rt.acc[0][n][2] * iv, rt.acc[0][n][3] * iv);
        }
        return;
    }
    if (!ok) return;
    bf16_t* o = (bf16_t*)a.o + (long long)(start + row) * a.o_tok + (long long)qh * a.o_head + h * 4;
#pragma unroll
    for (int n = 0; n < NHT; ++n)
#pragma unroll
        for (int u = 0; u < 4; ++u)
            *(bf16x4*)(o + n * 32 + u * 8) = E::pack4(acc[n][4 * u] * inv, acc[n][4 * u + 1] * inv, acc[n][4 * u + 2] * inv, acc[n][4 * u + 3] * inv);
}

}  // namespace

hipError_t launch_prompt_attention(int dtype, PromptArgs& a, const int32_t* cu, int n_seq, hipStream_t s) {
    // longest sequences first, in launches of as many as the kernel arguments hold
    std::vector<int> order;
    order.reserve(n_seq);
    for (int i = 0; i < n_seq; ++i)
        if (cu[i + 1] > cu[i]) order.push_back(i);
    std::stable_sort(order.begin(), order.end(), [&](int x, int y) { return cu[x + 1] - cu[x] > cu[y + 1] - cu[y]; });
    a.rows = dtype == 0 ? 16 : 128;
    a.cus = 256;
    for (size_t at = 0; at < order.size();) {
        const int n = (int)std::min<size_t>(order.size() - at, PROMPT_MAX_SEQ);
        for (int i = 0; i < n; ++i) {
            a.start[i] = cu[order[at + i]];
            a.len[i] = cu[order[at + i] + 1] - cu[order[at + i]];
        }
        at += n;
        const int blocks = (a.len[0] + a.rows - 1) / a.rows;  // of the longest sequence
        a.width = (blocks + PROMPT_MAX_SEQ - 1) / PROMPT_MAX_SEQ;
        a.levels = (blocks + a.width - 1) / a.width;
        long long units = 0;
        int with = 0;  // sequences that reach into the level
        for (int d = 0; d < a.levels; ++d) {
            a.first[d] = (int)units;
            while (with < n && a.len[with] > (long long)(a.levels - 1 - d) * a.width * a.rows) ++with;
            units += (long long)with * a.width;
        }
        if (units * a.Hq > 0x7fffffff) return hipErrorInvalidValue;
        a.units = (int)units * a.Hq;
        const dim3 grid(a.units);
        if (dtype == 0) {
            if (a.hd == 64) hipLaunchKernelGGL((prompt_rows_kernel<float, 64>), grid, dim3(256), 0, s, a);
            else hipLaunchKernelGGL((prompt_rows_kernel<float, 128>), grid, dim3(256), 0, s, a);
        } else {
            // Two groups of waves on alternate tiles where every block has a compute unit to itself and the longest row of tiles is what takes time
            // (16/8 heads of 64, 1000 tokens 17.2 -> 14.6 us, 2000 29.2 -> 23.9; 32 heads of 128, 1024 25.4 -> 24.5).  Up to 512 tokens the join costs
            // what it saves (two prompts of 512 17.3 -> 17.8, one of 100 8.1 -> 9.2), and with more blocks than units two workgroups of one group share
            // a unit better (2048 tokens, 512 blocks: 50.3 -> 59.5).
            const bool pair = a.units <= a.cus && a.len[0] > 512;
            if (a.hd == 64 && pair) hipLaunchKernelGGL((prompt_tiles_kernel<64, 2>), grid, dim3(512), 0, s, a);
            else if (a.hd == 64) hipLaunchKernelGGL((prompt_tiles_kernel<64, 1>), grid, dim3(256), 0, s, a);
            else if (pair) hipLaunchKernelGGL((prompt_tiles_kernel<128, 2>), grid, dim3(512), 0, s, a);
            else hipLaunchKernelGGL((prompt_tiles_kernel<128, 1>), grid, dim3(256), 0, s, a);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}
