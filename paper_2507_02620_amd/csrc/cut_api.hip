// Host side of the C ABI for sampling under cuts: validation, then a few launches.
#include <math.h>

#include "../../include/flowspec.h"
#include "cut.hpp"
#include "tree.hpp"

extern thread_local int g_last_hip;

#define HIP_TRY(expr)                 \
    do {                              \
        hipError_t e__ = (expr);      \
        if (e__ != hipSuccess) {      \
            g_last_hip = (int)e__;    \
            return FS_EHIP;           \
        }                             \
    } while (0)

static_assert(FS_SAMPLE_MAX_VOCAB == CUT_MAX_VOCAB, "header and kernels agree");

static bool valid_setting(float temperature, float top_p, float min_p) {
    return (temperature == 0.f || (temperature >= 0x1p-100f && temperature <= 0x1p100f)) && top_p == top_p && min_p == min_p;
}

extern "C" {

size_t fs_sample_workspace_bytes(int rows, int vocab) {
    if (rows < 1 || vocab < 1 || vocab > CUT_MAX_VOCAB || rows > FS_SAMPLE_MAX_ROWS) return 0;
    return accept_cut_bytes(rows) + 256 + cut_workspace_bytes(rows, vocab);
}

int fs_sample_tokens(int dtype, const void* logits, long long ld, int rows, int vocab, const fs_sampling* how, const double* u, int32_t* token,
                     float* logprob, int32_t* kept, void* workspace, size_t workspace_bytes, void* stream) {
    if (dtype != FS_F32 && dtype != FS_BF16) return FS_EDTYPE;
    if (rows < 0 || vocab < 1 || !how) return FS_EINVAL;
    if (vocab > CUT_MAX_VOCAB || rows > FS_SAMPLE_MAX_ROWS) return FS_ECAP;  // (rows: a launch's second dimension)
    if (!valid_setting(how->temperature ? 1.f : how->temperature_all, how->top_p ? 1.f : how->top_p_all, how->min_p ? 0.f : how->min_p_all)) return FS_EINVAL;
    if (rows == 0) return FS_OK;
    if (!logits || !u || !token || ld < vocab) return FS_EINVAL;
    if (((uintptr_t)logits & (dtype == FS_F32 ? 3 : 1)) || ((uintptr_t)u & 7)) return FS_EINVAL;
    if (((uintptr_t)how->temperature | (uintptr_t)how->top_k | (uintptr_t)how->top_p | (uintptr_t)how->min_p | (uintptr_t)token | (uintptr_t)logprob |
         (uintptr_t)kept) & 3)
        return FS_EINVAL;
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < fs_sample_workspace_bytes(rows, vocab)) return FS_EWS;
    CutArgs a{};
    a.logits = logits; a.ld = ld; a.rows = rows; a.vocab = vocab;
    a.how = CutSettings{how->temperature, how->top_k, how->top_p, how->min_p, how->temperature_all, how->top_k_all, how->top_p_all, how->min_p_all};
    a.u = u; a.token = token; a.logprob = logprob; a.kept = kept;
    HIP_TRY(launch_cut(dtype, a, workspace, (hipStream_t)stream));
    return FS_OK;
}

int fs_tree_accept_filtered(const float* logits, int vocab, float temperature, int top_k, float top_p, float min_p, const int32_t* token,
                            const int32_t* parent, int T, int n_ver, uint64_t seed, uint64_t step, fs_accept_result* res, int32_t* retain, void* workspace,
                            size_t workspace_bytes, void* stream) {
    if (!token || !parent || !res || !retain || T < 1 || n_ver < 0 || n_ver > T || vocab < 1) return FS_EINVAL;
    if (T > FS_MAX_TREE || vocab > CUT_MAX_VOCAB) return FS_ECAP;
    if (!(temperature > 0.f) || !valid_setting(temperature, top_p, min_p)) return FS_EINVAL;
    if (((uintptr_t)token | (uintptr_t)parent | (uintptr_t)res | (uintptr_t)retain | (uintptr_t)logits) & 3) return FS_EINVAL;
    if (n_ver > 0 && !logits) return FS_EINVAL;
    if (n_ver > 0 && (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < fs_sample_workspace_bytes(n_ver, vocab))) return FS_EWS;
    hipStream_t s = (hipStream_t)stream;
    RowCut* cuts = (RowCut*)workspace;
    if (n_ver > 0) {
        CutArgs a{};
        a.logits = logits; a.ld = vocab; a.rows = n_ver; a.vocab = vocab;
        a.how = CutSettings{nullptr, nullptr, nullptr, nullptr, temperature, top_k, top_p, min_p};
        a.cut = cuts;
        HIP_TRY(launch_cut(FS_F32, a, (char*)workspace + (accept_cut_bytes(n_ver) + 255) / 256 * 256, s));
    }
    HIP_TRY(launch_accept_cut(logits, vocab, 1.0f / temperature, token, parent, T, n_ver, seed, step, (AcceptResultDev*)res, retain, cuts, s));
    return FS_OK;
}

}  // extern "C"
