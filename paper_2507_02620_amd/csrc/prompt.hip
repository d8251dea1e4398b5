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

// Any type: a wave per 16 rows, keys and values from memory (L2) in halves of 32 slots, no workgroup-wide step at all.
template <typename T, int HD>
__global__ void __launch_bounds__(256) prompt_rows_kernel(const PromptArgs a) {
    using RT = RowTiles<T, HD, 1>;
    __shared__ __align__(16) T lds[4 * RT::STAGE];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), r16 = lane & 15, g = lane >> 4;
    const int b = a.blocks - 1 - (int)blockIdx.x, qh = blockIdx.y, kvh = qh / a.G;
    const int sq = seq_of(a, b), start = a.start[sq], len = a.len[sq];
    const int r0 = (b - a.block0[sq]) * 64 + w * 16;
    if (r0 >= len) return;  // no step of the workgroup as a whole follows
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
        if (s0 + 32 <= r0 + 1) rt.template half<false>(kp, vp, a.k_tok, a.v_tok, 31, vis, a.scale_log2, lds + w * RT::STAGE, lane);
        else rt.template half<true>(kp, vp, a.k_tok, a.v_tok, min(31, len - 1 - s0), vis, a.scale_log2, lds + w * RT::STAGE, lane);
    }
    const float inv = 1.0f / rt.row_sum(0);
    if (!ok) return;
    T* o = (T*)a.o + (long long)(start + r0 + r16) * a.o_tok + (long long)qh * a.o_head + g * 4;
#pragma unroll
    for (int n = 0; n < HD / 16; ++n)
        *(typename RT::E::out4_t*)(o + n * 16) =
            RT::E::pack4(rt.acc[0][n][0] * inv, rt.acc[0][n][1] * inv, rt.acc[0][n][2] * inv, rt.acc[0][n][3] * inv);
}

}  // namespace

hipError_t launch_prompt_attention(int dtype, PromptArgs& a, const int32_t* cu, int n_seq, hipStream_t s) {
    // longest sequences first, in launches of as many as the kernel arguments hold
    std::vector<int> order(n_seq);
    std::iota(order.begin(), order.end(), 0);
    std::stable_sort(order.begin(), order.end(), [&](int x, int y) { return cu[x + 1] - cu[x] > cu[y + 1] - cu[y]; });
    const int block = 64;
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
            if (a.hd == 64) hipLaunchKernelGGL((prompt_rows_kernel<bf16_t, 64>), grid, dim3(256), 0, s, a);
            else hipLaunchKernelGGL((prompt_rows_kernel<bf16_t, 128>), grid, dim3(256), 0, s, a);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}
