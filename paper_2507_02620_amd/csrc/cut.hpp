// Sampling under temperature, top-k, top-p and min-p: launch interface (see cut.hip).
#pragma once
#include "weights.hpp"

constexpr int CUT_MAX_VOCAB = 1 << 20;

// What is kept of a row: the scores before (z, idx) in the order z descending, index ascending, this one included, that weigh at least
// `least`.  R: the sum of their weights; 0 where a row has nothing to draw.
struct RowCut {
    float m;         // the row's largest score
    float z;
    unsigned idx;
    unsigned least_lo, least_hi;
    unsigned pad;
    uint64_t R;
};

// Weight of a score under the row's largest (above -inf): exp_weight's steps with the scaling as one exact ldexp and one conversion, a third less
// of a pass over weights; and scores equal to an infinite maximum share all of the mass.
static __device__ __forceinline__ uint64_t score_weight(float z, float m) {
    float t = fmaxf(mul_once(sub_once(z, m), 1.44269504088896341f), -64.0f);  // (what is not a number: -64, which weighs nothing)
    t = z == m ? 0.f : t;
    const float n = floorf(t), f = sub_once(t, n);
    float p = 1.52527338e-5f;
    p = fmaf(p, f, 1.54035304e-4f);
    p = fmaf(p, f, 1.33335581e-3f);
    p = fmaf(p, f, 9.61812911e-3f);
    p = fmaf(p, f, 5.55041087e-2f);
    p = fmaf(p, f, 2.40226507e-1f);
    p = fmaf(p, f, 6.93147181e-1f);
    p = fmaf(p, f, 1.0f);
    const float x = ldexpf(p, (int)n + 32);  // at most 2^32
    return x >= 0x1p32f ? 1ull << 32 : (uint64_t)(unsigned)x;
}

static __device__ __forceinline__ uint64_t cut_weight(const RowCut& c, float z, unsigned v) {
    if (!(z > c.z || (z == c.z && v <= c.idx))) return 0;
    const uint64_t w = score_weight(z, c.m);
    return w >= ((uint64_t)c.least_hi << 32 | c.least_lo) ? w : 0;
}

// One row of settings: a pointer per setting, or a value for all rows where it is null.
struct CutSettings {
    const float* temperature;
    const int32_t* top_k;
    const float *top_p, *min_p;
    float temperature_all;
    int32_t top_k_all;
    float top_p_all, min_p_all;
};

struct CutArgs {
    const void* logits;
    long long ld;  // elements between rows
    int rows, vocab;
    CutSettings how;
    const double* u;  // null: no draw, the rows' cuts only
    int32_t* token;
    float* logprob;   // or null
    int32_t* kept;    // or null
    RowCut* cut;      // or null
};

hipError_t launch_cut(int dtype, const CutArgs& a, void* work, hipStream_t s);
size_t cut_workspace_bytes(int rows, int vocab);

struct AcceptResultDev;
size_t accept_cut_bytes(int n_ver);
hipError_t launch_accept_cut(const float* logits, int vocab, float inv_temp, const int32_t* token, const int32_t* parent, int T, int n_ver, uint64_t seed,
                             uint64_t step, AcceptResultDev* res, int32_t* retain, RowCut* cuts /* accept_cut_bytes */, hipStream_t s);
