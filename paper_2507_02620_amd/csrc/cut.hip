// Sampling of a token per row under temperature, top-k, top-p and min-p, and the same cuts for acceptance along a tree.
//
// Scores z = logit * (1 / temperature) are rounded once to 32 bits; weights are the whole numbers of exp_weight, so sums have no order and
// every comparison is exact.  Order of a row: z descending, index ascending.  top-k keeps its first k; S is their sum; top-p keeps the
// shortest part whose sum reaches ceil(P S / 2^30), P = floor(p 2^30); min-p what weighs at least ceil(min_p 2^32).  The token is the first kept
// one by index whose running sum exceeds floor(U R / 2^48), R the sum of what is kept, U = floor(u 2^48).
#include "cut.hpp"

#include <algorithm>

namespace {

constexpr int THREADS = 1024, WAVES = THREADS / 64;

template <typename T>
static __device__ __forceinline__ float logit(const T* p, int i) {
    return (float)p[i];
}

// The settings of one row; ok: false where one of them is out of its range.
struct Setting {
    float inv;
    unsigned k;  // 0: all
    unsigned P;  // 2^30: all
    uint64_t least;
    bool ok;
};
static __device__ __forceinline__ Setting setting_of(const CutSettings& h, int row) {
    const float t = h.temperature ? h.temperature[row] : h.temperature_all, p = h.top_p ? h.top_p[row] : h.top_p_all,
                mp = h.min_p ? h.min_p[row] : h.min_p_all;
    const int k = h.top_k ? h.top_k[row] : h.top_k_all;
    Setting s;
    s.ok = (t == 0.f || (t >= 0x1p-100f && t <= 0x1p100f)) && p == p && mp == mp;
    s.inv = t == 0.f ? 1.f : 1.0f / t;
    s.k = t == 0.f ? 1u : k > 0 ? (unsigned)k : 0u;
    s.P = (unsigned)((double)fminf(fmaxf(p, 0.f), 1.f) * 0x1p30);
    s.least = max((uint64_t)ceil((double)fminf(fmaxf(mp, 0.f), 1.f) * 0x1p32), (uint64_t)1);
    return s;
}

// Keys that ascend along the order of a row (what is not a number comes last; -0 is 0).
static __device__ __forceinline__ unsigned down_key(float z) { return z == z ? ~max_key(z + 0.f) : ~0u; }
static __device__ __forceinline__ float key_score(unsigned kd) { return key_max(~kd); }

// a S / 2^bits, rounded down, of a < 2^bits
static __device__ __forceinline__ uint64_t part_of(uint64_t a, uint64_t s, int bits) { return (__umul64hi(a, s) << (64 - bits)) | ((a * s) >> bits); }
static __device__ __forceinline__ uint64_t top_p_need(unsigned P, uint64_t S) {
    const uint64_t n = S - part_of((1u << 30) - P, S, 30);  // ceil(P S / 2^30)
    return n > 1 ? n : 1;
}

// The element of a set at which the running count, or sum of weights, along the keys' order first reaches `need`.
struct Bound {
    uint64_t key;  // (down_key, index), or the index alone
    uint64_t sum;  // weights up to and with it
    unsigned count;
};
struct SelectLds {
    unsigned cnt[256];
    unsigned long long wt[256];
    unsigned digit;
    unsigned long long sum;
    unsigned count;
};

// Digit by digit of 8 bits from the highest on: each pass counts the elements that share the digits found so far.  each(fn) calls
// fn(key, weight) for all elements, in any order.  The set holds at least `need`.
template <bool BY_COUNT, typename Each>
static __device__ Bound select(SelectLds& l, int bits, uint64_t need, Each&& each) {
    Bound b{0, 0, 0};
    for (int sh = bits - 8; sh >= 0; sh -= 8) {
        __syncthreads();
        if (threadIdx.x < 256) {
            l.cnt[threadIdx.x] = 0;
            l.wt[threadIdx.x] = 0;
        }
        __syncthreads();
        const uint64_t prefix = b.key;
        each([&](uint64_t key, uint64_t w) {
            if (sh + 8 < bits && (key >> (sh + 8)) != prefix) return;
            const unsigned d = (unsigned)(key >> sh) & 255;
            atomicAdd(&l.cnt[d], 1u);
            atomicAdd(&l.wt[d], (unsigned long long)w);
        });
        __syncthreads();
        if (threadIdx.x < 64) {  // the first digit that reaches the need
            const int lane = threadIdx.x;
            uint64_t c[4], s[4], ct = 0, st = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                c[i] = l.cnt[lane * 4 + i];
                s[i] = l.wt[lane * 4 + i];
                ct += c[i];
                st += s[i];
            }
            uint64_t cb = wave_scan_u64(ct) - ct + b.count, sb = wave_scan_u64(st) - st + b.sum;  // before the lane's first digit
            const bool here = (BY_COUNT ? cb + ct : sb + st) >= need;
            const unsigned long long hit = __ballot(here);
            if (hit && lane == __ffsll(hit) - 1) {
                int i = 0;
                while (i < 3 && (BY_COUNT ? cb + c[i] : sb + s[i]) < need) {
                    cb += c[i];
                    sb += s[i];
                    ++i;
                }
                l.digit = lane * 4 + i;
                l.sum = sh ? sb : sb + s[i];
                l.count = (unsigned)(sh ? cb : cb + c[i]);
            }
        }
        __syncthreads();
        b.key = prefix << 8 | l.digit;
        b.sum = l.sum;
        b.count = l.count;
    }
    return b;
}

template <typename V, typename F>
static __device__ __forceinline__ V block_reduce(V v, V* sh, F&& f) {  // ends with a barrier
    for (int o = 32; o > 0; o >>= 1) v = f(v, __shfl_xor(v, o, FS_WAVE));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    v = sh[0];
    for (int w = 1; w < (int)blockDim.x / 64; ++w) v = f(v, sh[w]);
    __syncthreads();
    return v;
}

// One workgroup per row, everything by selection over the row in memory.
template <typename T>
__global__ void __launch_bounds__(THREADS) cut_row_kernel(const CutArgs a) {
    __shared__ SelectLds l;
    __shared__ uint64_t red[WAVES];
    const int row = blockIdx.x, tid = threadIdx.x, vocab = a.vocab;
    const T* p = (const T*)a.logits + (size_t)row * a.ld;
    const Setting s = setting_of(a.how, row);
    auto score = [&](int i) { return __fmul_rn(logit(p, i), s.inv); };
    float m = -INFINITY;
    for (int i = tid; i < vocab; i += THREADS) m = fmaxf(m, score(i));
    m = block_reduce(m, (float*)red, [](float x, float y) { return fmaxf(x, y); });
    const bool any = s.ok && m > -INFINITY;
    RowCut c{m, -INFINITY, ~0u, (unsigned)s.least, (unsigned)(s.least >> 32), 0, 0};
    uint64_t R = 0;
    unsigned kept = 0;
    if (any) {
        auto ordered = [&](auto&& fn) {  // what the order's cuts so far keep
            for (int i = tid; i < vocab; i += THREADS) {
                const float z = score(i);
                const uint64_t w = score_weight(z, m);
                if (w && (z > c.z || (z == c.z && (unsigned)i <= c.idx))) fn((uint64_t)down_key(z) << 24 | (unsigned)i, w);
            }
        };
        auto sum = [&](auto&& over, unsigned& n) {
            uint64_t w = 0;
            unsigned k = 0;
            over([&](uint64_t, uint64_t x) {
                w += x;
                ++k;
            });
            n = block_reduce(k, (unsigned*)red, [](unsigned x, unsigned y) { return x + y; });
            return block_reduce(w, red, [](uint64_t x, uint64_t y) { return x + y; });
        };
        unsigned n;
        uint64_t S = sum(ordered, n);
        if (s.k && s.k < n) {
            const Bound b = select<true>(l, 56, s.k, ordered);
            c.z = key_score((unsigned)(b.key >> 24));
            c.idx = (unsigned)b.key & 0xFFFFFF;
            S = b.sum;
        }
        if (s.P < (1u << 30)) {
            const Bound b = select<false>(l, 56, top_p_need(s.P, S), ordered);
            c.z = key_score((unsigned)(b.key >> 24));
            c.idx = (unsigned)b.key & 0xFFFFFF;
        }
        auto by_index = [&](auto&& fn) {
            for (int i = tid; i < vocab; i += THREADS) {
                const uint64_t w = cut_weight(c, score(i), i);
                if (w) fn((uint64_t)i, w);
            }
        };
        R = sum(by_index, kept);
        if (a.u) {
            const double u = a.u[row];
            const uint64_t U = !(u > 0.0) ? 0 : u >= 1.0 ? (1ull << 48) - 1 : (uint64_t)(u * 0x1p48);
            const Bound b = select<false>(l, 24, part_of(U, R, 48) + 1, by_index);
            if (tid == 0) {
                a.token[row] = (int)b.key;
                if (a.logprob) a.logprob[row] = (float)log((double)cut_weight(c, score((int)b.key), (unsigned)b.key) / (double)R);
                if (a.kept) a.kept[row] = (int)kept;
            }
        }
    } else if (a.u && tid == 0) {
        a.token[row] = -1;
        if (a.logprob) a.logprob[row] = -INFINITY;
        if (a.kept) a.kept[row] = 0;
    }
    if (a.cut && tid == 0) {
        c.R = R;
        a.cut[row] = c;
    }
}

}  // namespace

size_t cut_workspace_bytes(int rows, int vocab) { return ((size_t)rows * sizeof(RowCut) + 255) / 256 * 256; }

hipError_t launch_cut(int dtype, const CutArgs& a, void* work, hipStream_t s) {
    if (dtype == 0) hipLaunchKernelGGL((cut_row_kernel<float>), dim3(a.rows), dim3(THREADS), 0, s, a);
    else hipLaunchKernelGGL((cut_row_kernel<bf16_t>), dim3(a.rows), dim3(THREADS), 0, s, a);
    return hipGetLastError();
}
