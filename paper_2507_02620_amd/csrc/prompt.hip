// Causal attention over whole prompts packed behind one another, grouped heads.
#include "paged.hpp"
#include "rows_attn.hpp"

#include <algorithm>
#include <numeric>
#include <vector>

namespace {

// The sequence that owns block b of the launch (block0 ascending, block0[n_seq] = blocks).
static __device__ __forceinline__ int seq_of(const PromptArgs& a, int b) {
    int lo = 0, hi = a.n_seq - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (a.block0[mid] <= b) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// 16 rows of a sequence by one wave, keys and values from memory (L2) in halves of 32 slots, no workgroup-wide step at all.
template <typename T, int HD>
static __device__ __forceinline__ void rows16(const PromptArgs& a, int start, int len, int r0, int qh, T* vt, int lane) {
    using RT = RowTiles<T, HD, 1>;
    const int r16 = lane & 15, g = lane >> 4, kvh = qh / a.G;
    RT rt;
    rt.init();
    const bool ok = r0 + r16 < len;
    rt.load_q(0, (const T*)a.q + (long long)(start + (ok ? r0 + r16 : r0)) * a.q_tok + (long long)qh * a.q_head, ok, g);
    const T* kb = (const T*)a.k + (long long)start * a.k_tok + (long long)kvh * a.k_head;
    const T* vb = (const T*)a.v + (long long)start * a.v_tok + (long long)kvh * a.v_head;
    const int end = min(len, r0 + 16);  // slots the wave's last row sees
    for (int s0 = 0; s0 < end; s0 += 32) {
        const int n = r0 + r16 + 1 - s0;
        unsigned vis[1] = {!ok || n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1};
        const T *kp = kb + (long long)s0 * a.k_tok, *vp = vb + (long long)s0 * a.v_tok;
        if (s0 + 32 <= r0 + 1) rt.template half<false>(kp, vp, a.k_tok, a.v_tok, 31, vis, a.scale_log2, vt, lane);
        else rt.template half<true>(kp, vp, a.k_tok, a.v_tok, min(31, len - 1 - s0), vis, a.scale_log2, vt, lane);
    }
    const float inv = 1.0f / rt.row_sum(0);
    if (!ok) return;
    T* o = (T*)a.o + (long long)(start + r0 + r16) * a.o_tok + (long long)qh * a.o_head + g * 4;
#pragma unroll
    for (int n = 0; n < HD / 16; ++n)
        *(typename RT::E::out4_t*)(o + n * 16) =
            RT::E::pack4(rt.acc[0][n][0] * inv, rt.acc[0][n][1] * inv, rt.acc[0][n][2] * inv, rt.acc[0][n][3] * inv);
}

// f32: a workgroup per 64 rows of a head.
template <typename T, int HD>
__global__ void __launch_bounds__(256) prompt_rows_kernel(const PromptArgs a) {
    constexpr int STAGE = RowTiles<T, HD, 1>::STAGE;
    __shared__ __align__(16) T lds[4 * STAGE];
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int b = a.blocks - 1 - (int)blockIdx.x, sq = seq_of(a, b), r0 = (b - a.block0[sq]) * 64 + w * 16;
    if (r0 < a.len[sq]) rows16<T, HD>(a, a.start[sq], a.len[sq], r0, blockIdx.y, lds + w * STAGE, threadIdx.x & 63);
}

// bf16: a workgroup per 128 rows of a head, a wave per 32.
//
// S^T = K . Q^T and O^T += V^T . P^T by 32x32x16 products: lane l holds values of query row l % 32 only (two lanes to a row), so the
// softmax state is per lane and P never leaves registers: S^T has slot 8 (v / 4) + 4 (l / 32) + v % 4 in register v, which is
// the order in which the V^T operand is read with the transposing LDS load.  K/V tiles of 64 slots go from memory straight into LDS, two
// buffers, one barrier per tile, the 16-byte chunk c of row r at chunk c ^ (r mod chunks) so that neither read meets bank conflicts.
// Two workgroups share a compute unit: one's exponentials run behind the other's matrix products.
//
// The running maximum is only raised where a score exceeds it by more than 2^8 in the exponential (any common factor of numerator and
// denominator is as good; 8 bits of headroom cost no precision in floating point), so most tiles rescale nothing.
// A masked slot's V row is multiplied by zero, which a value that is not finite would survive: a wave that ends with any such sum does
// its rows again slot by slot.
typedef float f32x16 __attribute__((ext_vector_type(16)));

template <int HD>
__global__ void __launch_bounds__(512) prompt_tiles_kernel(int units, const PromptArgs a) {
    using E = Elem<bf16_t>;
    constexpr int BS = 64, ROWB = HD * 2, CHUNKS = ROWB / 16, NKT = HD / 16, NHT = HD / 32, TILE = BS * ROWB;
    constexpr int RPL = 1024 / ROWB, LPW = BS / RPL / 4;  // rows per direct-to-LDS load of a wave; such loads per wave and tile (K, and V)
    constexpr float HEADROOM = 8.f;
    __shared__ __align__(1024) unsigned char tb0[2 * TILE];
    __shared__ __align__(1024) unsigned char tb1[2 * TILE];
    constexpr int STAGE = RowTiles<bf16_t, HD, 1>::STAGE;
    static_assert(2 * STAGE * 2 <= 2 * TILE, "two waves' stages fit one buffer");

    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), c32 = lane & 31, h = lane >> 5;
    // ---- which rows ----
    int b, qh;
    {
        const int id = blockIdx.x;
        b = a.blocks - 1 - id / a.Hq;
        qh = id % a.Hq;
    }
    const int sq = seq_of(a, b), start = a.start[sq], len = a.len[sq], kvh = qh / a.G;
    const int blk0 = (b - a.block0[sq]) * 128, r0 = blk0 + w * 32, row = r0 + c32;
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
    const unsigned kst = (unsigned)a.k_tok * 2, vst = (unsigned)a.v_tok * 2;
    // load i of a wave brings rows RPL (LPW w + i) + lane / CHUNKS; rows behind the sequence re-read its last one (they are masked)
    auto issue = [&](int t, unsigned char* buf) __attribute__((always_inline)) {
        const int last = len - 1 - t * BS;
        const unsigned char *kt = kb + (long long)t * BS * a.k_tok * 2, *vt = vb + (long long)t * BS * a.v_tok * 2;
#pragma unroll
        for (int i = 0; i < LPW; ++i) {
            const int r = RPL * (LPW * w + i) + lane / CHUNKS;
            const unsigned col = (unsigned)(((lane % CHUNKS) ^ (r % CHUNKS)) * 16);
            __builtin_amdgcn_global_load_lds(FS_GLB_PTR(kt + ((unsigned)min(r, last) * kst + col)), FS_LDS_PTR(buf + RPL * (LPW * w + i) * ROWB), 16, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < LPW; ++i) {
            const int r = RPL * (LPW * w + i) + lane / CHUNKS;
            const unsigned col = (unsigned)(((lane % CHUNKS) ^ (r % CHUNKS)) * 16);
            __builtin_amdgcn_global_load_lds(FS_GLB_PTR(vt + ((unsigned)min(r, last) * vst + col)), FS_LDS_PTR(buf + TILE + RPL * (LPW * w + i) * ROWB), 16, 0, 0);
        }
    };
    unsigned kread[NKT], vread[NHT][2];
#pragma unroll
    for (int kt = 0; kt < NKT; ++kt) kread[kt] = (unsigned)(c32 * ROWB + (((kt * 2 + h) ^ (c32 % CHUNKS)) * 16));
    {
        const int i = lane & 15, sub = (lane >> 4) & 1;
#pragma unroll
        for (int n = 0; n < NHT; ++n)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int r = 8 * u + 4 * h + (i >> 2);
                vread[n][u] = (unsigned)(TILE + r * ROWB + (((n * 4 + sub * 2 + ((i & 3) >> 1)) ^ (r % CHUNKS)) * 16) + (i & 1) * 8);
            }
    }

    auto process = [&](int t, const unsigned char* buf) __attribute__((always_inline)) {
        const int s0 = t * BS;
        if (s0 > r0 + 31 || r0 >= len) return;  // wave-uniform: behind the wave's last row, or it has none
        f32x16 st[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
#pragma unroll
            for (int v = 0; v < 16; ++v) st[s][v] = 0.f;
#pragma unroll
            for (int kt = 0; kt < NKT; ++kt)
                st[s] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const bf16x8*)(buf + kread[kt] + s * 32 * ROWB), qf[kt], st[s], 0, 0, 0);
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
        mx = wave_xor_max(mx, 32) * a.scale_log2;
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
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(st[s][v], a.scale_log2, -ms));
                st[s][v] = e;
                sum += e;
            }
        l += sum;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            bf16x8 pf;
#pragma unroll
            for (int e = 0; e < 8; ++e) pf[e] = (bf16_t)st[c / 2][(c % 2) * 8 + e];
#pragma unroll
            for (int n = 0; n < NHT; ++n) {
                const s16x4 x0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(buf + vread[n][0] + c * 16 * ROWB));
                const s16x4 x1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(buf + vread[n][1] + c * 16 * ROWB));
                const bf16x8 vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(x0, x1, 0, 1, 2, 3, 4, 5, 6, 7));
                acc[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf, acc[n], 0, 0, 0);
            }
        }
    };

    issue(0, tb0);
    auto step = [&](int t, unsigned char* buf, unsigned char* other) __attribute__((always_inline)) {
        asm volatile("" ::: "memory");
        FS_WAIT_VM_LGKM(0, 0);
        __builtin_amdgcn_s_barrier();  // the tile is complete for every wave; every wave is done with the one before it
        asm volatile("" ::: "memory");
        if (t + 1 < tiles) issue(t + 1, other);
        process(t, buf);
    };
    for (int t = 0; t < tiles; t += 2) {
        step(t, tb0, tb1);
        if (t + 1 < tiles) step(t + 1, tb1, tb0);
    }

    l = wave_xor_add(l, 32);
    const float inv = 1.0f / l;
    bool odd = !(fabsf(l) < __builtin_inff());
#pragma unroll
    for (int n = 0; n < NHT; ++n)
#pragma unroll
        for (int v = 0; v < 16; ++v) odd |= !(fabsf(acc[n][v]) < __builtin_inff());
    const bool again = __ballot(ok && odd) != 0;
    __syncthreads();  // both buffers are free
    if (again) {
#pragma nounroll
        for (int i = 0; i < 2; ++i)
            if (r0 + 16 * i < len) rows16<bf16_t, HD>(a, start, len, r0 + 16 * i, qh, (bf16_t*)(w < 2 ? tb0 : tb1) + (w & 1) * STAGE, lane);
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
    std::vector<int> order(n_seq);
    std::iota(order.begin(), order.end(), 0);
    std::stable_sort(order.begin(), order.end(), [&](int x, int y) { return cu[x + 1] - cu[x] > cu[y + 1] - cu[y]; });
    const int block = dtype == 0 ? 64 : 128;
    for (int at = 0; at < n_seq;) {
        a.n_seq = 0;
        a.blocks = 0;
        for (; at < n_seq && a.n_seq < PROMPT_MAX_SEQ; ++at) {
            const int x = order[at], len = cu[x + 1] - cu[x];
            if (len == 0) continue;
            a.start[a.n_seq] = cu[x];
            a.len[a.n_seq] = len;
            a.block0[a.n_seq++] = a.blocks;
            a.blocks += (len + block - 1) / block;
        }
        a.block0[a.n_seq] = a.blocks;
        if (a.blocks == 0) break;
        const dim3 grid(a.blocks, a.Hq);
        if (dtype == 0) {
            if (a.hd == 64) hipLaunchKernelGGL((prompt_rows_kernel<float, 64>), grid, dim3(256), 0, s, a);
            else hipLaunchKernelGGL((prompt_rows_kernel<float, 128>), grid, dim3(256), 0, s, a);
        } else {
            const int units = a.blocks * a.Hq;
            if (a.hd == 64) hipLaunchKernelGGL((prompt_tiles_kernel<64>), dim3(units), dim3(256), 0, s, units, a);
            else hipLaunchKernelGGL((prompt_tiles_kernel<128>), dim3(units), dim3(256), 0, s, units, a);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}
