// Sampling of a token per row under temperature, top-k, top-p and min-p, and the same cuts for acceptance along a tree.
//
// Scores z = logit * (1 / temperature) are rounded once to 32 bits; weights are the whole numbers of exp_weight, so sums have no order and
// every comparison is exact.  Order of a row: z descending, index ascending.  top-k keeps its first k; S is their sum; top-p keeps the
// shortest part whose sum reaches ceil(P S / 2^30), P = floor(p 2^30); min-p what weighs at least ceil(min_p 2^32).  The token is the first kept
// one by index whose running sum exceeds floor(U R / 2^48), R the sum of what is kept, U = floor(u 2^48).
#include "cut.hpp"

#include <algorithm>

namespace {

template <typename T>
static __device__ __forceinline__ float logit(const T* p, int i) {
    return (float)p[i];
}

// Four consecutive logits.
template <typename T>
static __device__ __forceinline__ f32x4 logits4(const T* p) {
    const typename Elem<T>::out4_t x = *(const typename Elem<T>::out4_t*)p;
    return f32x4{Elem<T>::to_f(x[0]), Elem<T>::to_f(x[1]), Elem<T>::to_f(x[2]), Elem<T>::to_f(x[3])};
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

// ---- bins: scores by their distance from the row's largest ---------------------------------------------------------------------
// 64 bins to a power of two of the distance d = fl(m - z), from 2^-20 on; bin 0 is what lies nearer.  d falls as z rises, so bins keep the order.
// Weights end at d = 32 ln 2 = 22.2.  Relative bins suit every scale of scores: of N(0, s^2) rows the fullest one holds 2.6 % whatever s.
constexpr unsigned D0 = 0x35800000u;  // 2^-20
constexpr int BIN_SHIFT = 17, BINS = 1600;
static __device__ __forceinline__ unsigned dist_bits(float z, float m) { return z == m ? 0u : __float_as_uint(__fsub_rn(m, z)); }
static __device__ __forceinline__ int bin_of(unsigned d) { return d < D0 ? 0 : min((int)((d - D0) >> BIN_SHIFT) + 1, BINS - 1); }

// ---- selection -------------------------------------------------------------------------------------------------------------------
// Counts and weights of bins or digits; `find` sees them in order.
struct Tally {
    unsigned long long mass[BINS];
    unsigned cnt[BINS];
};
struct Found {
    int bin;            // the first one with which the running count, or weight, reaches the need; n if none does
    unsigned cnt, in_cnt;  // before it; in it
    uint64_t mass, in_mass;
};
constexpr int DIGIT = 10;
template <int NT>
struct CutLds {
    unsigned long long mass[1 << DIGIT];
    unsigned cnt[1 << DIGIT];
    unsigned long long wm[NT / 64];
    unsigned wc[NT / 64];
    unsigned long long red[NT / 64];
    Found found;
    unsigned zmin, zmax;
    float z1;
    unsigned i1;
};

// Block-wide, with a barrier before and behind: bins [0, n) of any arrays.
template <int NT, typename L>
static __device__ Found find(L& l, const unsigned long long* mass, const unsigned* cnt, int n, uint64_t need, bool by_count, unsigned cnt0, uint64_t mass0) {
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, each = (n + NT - 1) / NT, lo = min(n, tid * each), hi = min(n, lo + each);
    __syncthreads();
    unsigned c = 0;
    uint64_t m = 0;
    for (int i = lo; i < hi; ++i) {
        c += cnt[i];
        m += mass[i];
    }
    unsigned cs = c;
    uint64_t ms = m;
    for (int o = 1; o < 64; o <<= 1) {
        const unsigned cu = __shfl_up(cs, o, FS_WAVE);
        const uint64_t mu = __shfl_up(ms, o, FS_WAVE);
        if (lane >= o) {
            cs += cu;
            ms += mu;
        }
    }
    if (lane == 63) {
        l.wc[w] = cs;
        l.wm[w] = ms;
    }
    if (tid == 0) l.found.bin = n;
    __syncthreads();
    unsigned cb = cnt0 + cs - c, ct = cnt0;
    uint64_t mb = mass0 + ms - m, mt = mass0;
#pragma unroll
    for (int k = 0; k < NT / 64; ++k) {
        cb += k < w ? l.wc[k] : 0;
        mb += k < w ? l.wm[k] : 0;
        ct += l.wc[k];
        mt += l.wm[k];
    }
    if (by_count ? cb < need && cb + c >= need : mb < need && mb + m >= need) {  // one thread
        int i = lo;
        for (; i + 1 < hi && (by_count ? cb + cnt[i] : mb + mass[i]) < need; ++i) {
            cb += cnt[i];
            mb += mass[i];
        }
        l.found = Found{i, cb, cnt[i], mb, mass[i]};
    }
    __syncthreads();
    Found f = l.found;
    if (f.bin == n) f = Found{n, ct, 0, mt, 0};
    return f;
}

// The last element that is kept: of those in bin b, the one at which the running count (or weight) along the order, `f` before the bin, first
// reaches the need.  Digits of ten bits of d, then of z's key, then of the index, until one element is left.  each(fn) calls fn(z, index) for the
// elements of the row, or at least for all of that bin, in any order.
struct Bound {
    float z;
    unsigned idx;
    unsigned cnt;   // up to and with it
    uint64_t mass;
};
template <int NT, typename L, typename Each>
static __device__ Bound select_in(L& l, float m, Found f, uint64_t need, bool by_count, Each&& each) {
    const int tid = threadIdx.x, bin = f.bin;
    unsigned d_at = 0, z_at = 0, i_at = 0;  // digits found so far
    int d_sh = bin ? BIN_SHIFT : 30, z_sh = 32, i_sh = 20;
    if (bin) d_at = (D0 >> BIN_SHIFT) + bin - 1;
    auto member = [&](float z, unsigned i, unsigned& d, unsigned& k) {
        d = dist_bits(z, m);
        k = down_key(z);
        if ((uint64_t)d >> d_sh != d_at || (bin == 0 && d >= D0)) return false;
        return d_sh > 0 || ((uint64_t)k >> z_sh == z_at && (z_sh > 0 || i >> i_sh == i_at));
    };
    while (f.in_cnt > 1 && (d_sh | z_sh | i_sh)) {
        if (d_sh == 0 && z_sh == 32) {  // the same distance: mostly the same score
            __syncthreads();
            if (tid == 0) {
                l.zmin = ~0u;
                l.zmax = 0u;
            }
            __syncthreads();
            each([&](float z, unsigned i) {
                unsigned d, k;
                if (score_weight(z, m) && member(z, i, d, k)) {
                    atomicMin(&l.zmin, k);
                    atomicMax(&l.zmax, k);
                }
            });
            __syncthreads();
            if (l.zmin == l.zmax) {
                z_at = l.zmin;
                z_sh = 0;
                continue;
            }
        }
        const int level = d_sh ? 0 : z_sh ? 1 : 2, from = level == 0 ? d_sh : level == 1 ? z_sh : i_sh, to = max(from - DIGIT, 0), n = 1 << (from - to);
        __syncthreads();
        for (int i = tid; i < n; i += NT) {
            l.mass[i] = 0;
            l.cnt[i] = 0;
        }
        __syncthreads();
        each([&](float z, unsigned i) {
            unsigned d, k;
            if (!member(z, i, d, k)) return;
            const uint64_t w = score_weight(z, m);
            if (!w) return;
            const unsigned at = ((level == 0 ? d : level == 1 ? k : i) >> to) & (n - 1);
            atomicAdd(&l.cnt[at], 1u);
            atomicAdd(&l.mass[at], (unsigned long long)w);
        });
        f = find<NT>(l, l.mass, l.cnt, n, need, by_count, f.cnt, f.mass);
        if (level == 0) {
            d_at = d_at << (from - to) | f.bin;
            d_sh = to;
        } else if (level == 1) {
            z_at = z_at << (from - to) | f.bin;
            z_sh = to;
        } else {
            i_at = i_at << (from - to) | f.bin;
            i_sh = to;
        }
    }
    __syncthreads();
    each([&](float z, unsigned i) {
        unsigned d, k;
        if (member(z, i, d, k) && score_weight(z, m)) {  // one element
            l.z1 = z;
            l.i1 = i;
        }
    });
    __syncthreads();
    return Bound{l.z1, l.i1, f.cnt + f.in_cnt, f.mass + f.in_mass};
}

template <int NT, typename V, typename L, typename F>
static __device__ __forceinline__ V block_reduce(L& l, V v, F&& f) {  // ends with a barrier
    V* sh = (V*)l.red;
    for (int o = 32; o > 0; o >>= 1) v = f(v, __shfl_xor(v, o, FS_WAVE));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    v = sh[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) v = f(v, sh[w]);
    __syncthreads();
    return v;
}

static __device__ __forceinline__ RowCut uncut(const Setting& s, float m) {
    return RowCut{m, -INFINITY, ~0u, (unsigned)s.least, (unsigned)(s.least >> 32), 0, 0};
}
static __device__ __forceinline__ uint64_t draw_target(const CutArgs& a, int row, uint64_t R) {
    const double u = a.u[row];
    return part_of(!(u > 0.0) ? 0 : u >= 1.0 ? (1ull << 48) - 1 : (uint64_t)(u * 0x1p48), R, 48);
}
static __device__ __forceinline__ void emit(const CutArgs& a, int row, int token, uint64_t w, uint64_t R, unsigned kept) {
    a.token[row] = token;
    if (a.logprob) a.logprob[row] = token < 0 ? -INFINITY : (float)log((double)w / (double)R);
    if (a.kept) a.kept[row] = (int)kept;
}

// The first of the block's NT * 4 consecutive entries (four of a thread's, w their weights) with which the running sum, `base` before them, exceeds
// the target; -1 if none does.  base becomes the sum behind them.  Two barriers.
template <int NT, typename L>
static __device__ __forceinline__ int first_over(L& l, const uint64_t (&w)[4], uint64_t& base, uint64_t target) {
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const uint64_t own = w[0] + w[1] + w[2] + w[3];
    const uint64_t run = wave_scan_u64(own);
    __syncthreads();
    if (lane == 63) l.red[wv] = run;
    if (tid == 0) l.i1 = ~0u;
    __syncthreads();
    uint64_t before = base;
#pragma unroll
    for (int k = 0; k < NT / 64; ++k) {
        before += k < wv ? l.red[k] : 0;
        base += l.red[k];
    }
    if (base <= target) return -1;
    before += run - own;
    if (before <= target && target < before + own) {
        int e = 0;
        while ((before += w[e]) <= target) ++e;
        l.i1 = tid * 4 + e;
    }
    __syncthreads();
    return (int)l.i1;
}

// Bins of a row, and what of it the cuts along the order keep: top-k, then top-p over what that leaves.
template <int NT, typename L, typename Each>
static __device__ void cut_along(L& l, const unsigned long long* mass, const unsigned* cnt, const Setting& s, Each&& each, RowCut& c) {
    uint64_t S = 0;
    if (s.k) {
        const Found f = find<NT>(l, mass, cnt, BINS, s.k, true, 0, 0);
        S = f.mass;
        if (f.bin < BINS) {
            const Bound b = select_in<NT>(l, c.m, f, s.k, true, each);
            c.z = b.z;
            c.idx = b.idx;
            S = b.mass;
        }
    } else {
        S = find<NT>(l, mass, cnt, BINS, ~0ull, false, 0, 0).mass;
    }
    if (s.P >= (1u << 30)) return;
    const uint64_t need = top_p_need(s.P, S);
    const Found f = find<NT>(l, mass, cnt, BINS, need, false, 0, 0);
    const Bound b = select_in<NT>(l, c.m, f, need, false, each);
    c.z = b.z;
    c.idx = b.idx;
}

// ---- a row per workgroup, its scores in LDS: one launch ----------------------------------------------------------------------
template <typename T, int NT, int MOST>
__global__ void __launch_bounds__(NT) cut_row_kernel(const CutArgs a, bool vec) {
    __shared__ CutLds<NT> l;
    __shared__ Tally t;
    __shared__ __align__(16) float z[MOST];
    const int row = blockIdx.x, tid = threadIdx.x, vocab = a.vocab;
    const T* p = (const T*)a.logits + (size_t)row * a.ld;
    const Setting s = setting_of(a.how, row);
    float m = -INFINITY;
    const int full = (vocab + 4 * NT - 1) & ~(4 * NT - 1);
    for (int i = tid * 4; i < full; i += NT * 4) {
        f32x4 x{NAN, NAN, NAN, NAN};  // (weighs nothing)
        if (vec && i + 4 <= vocab) x = logits4(p + i);
        else
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (i + e < vocab) x[e] = logit(p, i + e);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[e] = __fmul_rn(x[e], s.inv);
            m = fmaxf(m, x[e]);
        }
        *(f32x4*)(z + i) = x;
    }
    const bool along = s.k || s.P < (1u << 30);
    if (along)
        for (int i = tid; i < BINS; i += NT) {
            t.mass[i] = 0;
            t.cnt[i] = 0;
        }
    m = block_reduce<NT>(l, m, [](float x, float y) { return fmaxf(x, y); });
    RowCut c = uncut(s, m);
    const bool any = s.ok && m > -INFINITY;
    auto each = [&](auto&& fn) __attribute__((always_inline)) {
        for (int i = tid; i < vocab; i += NT) fn(z[i], (unsigned)i);
    };
    if (any && along) {
        each([&](float x, unsigned) {
            const uint64_t w = score_weight(x, m);
            if (!w) return;
            const int b = bin_of(dist_bits(x, m));
            atomicAdd(&t.cnt[b], 1u);
            atomicAdd(&t.mass[b], (unsigned long long)w);
        });
        cut_along<NT>(l, t.mass, t.cnt, s, each, c);
    }
    unsigned kept = 0;
    uint64_t R = 0;
    if (any) {
        each([&](float x, unsigned i) {
            const uint64_t w = cut_weight(c, x, i);
            R += w;
            kept += w != 0;
        });
        R = block_reduce<NT>(l, R, [](uint64_t x, uint64_t y) { return x + y; });
    }
    c.R = R;
    if (a.cut && tid == 0) a.cut[row] = c;
    if (!a.u) return;
    if (!any) {
        if (tid == 0) emit(a, row, -1, 0, 0, 0);
        return;
    }
    kept = block_reduce<NT>(l, kept, [](unsigned x, unsigned y) { return x + y; });
    const uint64_t target = draw_target(a, row, R);
    uint64_t base = 0;
    for (int i0 = 0; i0 < vocab; i0 += NT * 4) {
        const int i = i0 + tid * 4;
        const f32x4 x = *(const f32x4*)(z + i);
        uint64_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = cut_weight(c, x[e], i + e);
        const int at = first_over<NT>(l, w, base, target);
        if (at < 0) continue;
        if (at / 4 == tid) emit(a, row, i0 + at, at % 4 == 0 ? w[0] : at % 4 == 1 ? w[1] : at % 4 == 2 ? w[2] : w[3], R, kept);
        return;
    }
}

// ---- rows in chunks over the chip ---------------------------------------------------------------------------------------------------
// Four launches: the chunks' maxima; the bins; what lies in the bins that a cut passes through, to a list of the row's, beside what is surely kept, summed by
// chunk; and a workgroup per row that finds the cut in the list and the token in the chunk that the target falls into.
constexpr int CHUNKS = 64, LIST = 8192, CT = 256;
struct RowState {
    unsigned long long mass[BINS];
    unsigned cnt[BINS];
    unsigned listed, pad[3];
    unsigned long long chunk_mass[CHUNKS];
    unsigned chunk_cnt[CHUNKS];
    float chunk_max[CHUNKS];
    struct {
        float z;
        unsigned idx;
    } list[LIST];
};

template <typename T, typename F>
static __device__ __forceinline__ void for_chunk(const T* p, int lo, int hi, bool vec, F&& fn) {  // lo a multiple of 4
    int i = lo + threadIdx.x * 4;
    if (vec) {
        for (; i + 3 * CT * 4 + 4 <= hi; i += 4 * CT * 4) {  // four loads in flight
            f32x4 x[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = logits4(p + i + k * CT * 4);
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) fn(x[k][e], i + k * CT * 4 + e);
        }
    }
    for (; i < hi; i += CT * 4) {
        f32x4 x{NAN, NAN, NAN, NAN};
        if (vec && i + 4 <= hi) x = logits4(p + i);
        else
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (i + e < hi) x[e] = logit(p, i + e);
#pragma unroll
        for (int e = 0; e < 4; ++e) fn(x[e], i + e);
    }
}

template <typename T>
__global__ void __launch_bounds__(CT) chunk_max_kernel(const CutArgs a, RowState* __restrict__ st, int chunk, bool vec) {
    __shared__ float red[CT / 64];
    const int row = blockIdx.y, c = blockIdx.x, tid = threadIdx.x;
    RowState& r = st[row];
    for (int i = c * CT + tid; i < BINS; i += gridDim.x * CT) {  // for the launches behind this one
        r.mass[i] = 0;
        r.cnt[i] = 0;
    }
    if (c == 0 && tid == 0) r.listed = 0;
    const T* p = (const T*)a.logits + (size_t)row * a.ld;
    const int lo = c * chunk, hi = min(a.vocab, lo + chunk);
    const float inv = setting_of(a.how, row).inv;
    float m = -INFINITY;
    for_chunk(p, lo, hi, vec, [&](float x, int) { m = fmaxf(m, __fmul_rn(x, inv)); });
    for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, FS_WAVE));
    if ((tid & 63) == 0) red[tid >> 6] = m;
    __syncthreads();
    if (tid == 0) r.chunk_max[c] = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
}

static __device__ __forceinline__ float row_max(const RowState& r, int chunks) {  // every wave by itself
    float m = (int)(threadIdx.x & 63) < chunks ? r.chunk_max[threadIdx.x & 63] : -INFINITY;
    for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, FS_WAVE));
    return m;
}

template <typename T>
__global__ void __launch_bounds__(CT) chunk_bins_kernel(const CutArgs a, RowState* __restrict__ st, int chunk, bool vec) {
    __shared__ Tally t;
    const int row = blockIdx.y, tid = threadIdx.x;
    const Setting s = setting_of(a.how, row);
    if (!s.k && s.P >= (1u << 30)) return;  // no cut along the order
    RowState& r = st[row];
    const float m = row_max(r, gridDim.x);
    if (!s.ok || !(m > -INFINITY)) return;
    for (int i = tid; i < BINS; i += CT) {
        t.mass[i] = 0;
        t.cnt[i] = 0;
    }
    __syncthreads();
    const T* p = (const T*)a.logits + (size_t)row * a.ld;
    const int lo = blockIdx.x * chunk, hi = min(a.vocab, lo + chunk);
    for_chunk(p, lo, hi, vec, [&](float x, int) {
        const float z = __fmul_rn(x, s.inv);
        const uint64_t w = score_weight(z, m);
        if (!w) return;
        const int b = bin_of(dist_bits(z, m));
        atomicAdd(&t.cnt[b], 1u);
        atomicAdd(&t.mass[b], (unsigned long long)w);
    });
    __syncthreads();
    for (int i = tid; i < BINS; i += CT)
        if (t.cnt[i]) {
            atomicAdd(&r.cnt[i], t.cnt[i]);
            atomicAdd(&r.mass[i], t.mass[i]);
        }
}

// Which bins go to the list and which are kept for sure; the same for every workgroup of a row.
struct Plan {
    Found k;         // where top-k ends (k.bin == BINS: nowhere)
    int lo, hi;      // bins [lo, hi] and k.bin are listed; below lo everything is kept; lo == BINS: no cut
    bool listed_k, fits;
};
template <int NT, typename L>
static __device__ Plan plan_of(L& l, const RowState& r, const Setting& s) {
    const bool by_mass = s.P < (1u << 30);
    Plan p{Found{BINS, 0, 0, 0, 0}, BINS, BINS, false, true};
    if (!s.k && !by_mass) return p;
    if (s.k) p.k = find<NT>(l, r.mass, r.cnt, BINS, s.k, true, 0, 0);
    if (!by_mass) {
        p.lo = p.hi = p.k.bin;
        p.fits = p.k.in_cnt <= LIST;
        return p;
    }
    // top-p ends no later than if all of top-k's last bin counted, and no earlier than if none of it did
    uint64_t upto = p.k.mass + p.k.in_mass;
    if (!s.k) upto = find<NT>(l, r.mass, r.cnt, BINS, ~0ull, false, 0, 0).mass;
    const Found late = find<NT>(l, r.mass, r.cnt, BINS, top_p_need(s.P, upto), false, 0, 0);
    p.hi = p.lo = late.bin;
    unsigned n = late.in_cnt;
    if (p.k.bin < BINS) {
        const Found early = find<NT>(l, r.mass, r.cnt, BINS, top_p_need(s.P, p.k.mass), false, 0, 0);
        p.lo = early.bin < BINS ? early.bin : 0;
        n = late.cnt + late.in_cnt - (early.bin < BINS ? early.cnt : 0) + (p.k.bin > p.hi ? p.k.in_cnt : 0);
        p.listed_k = true;
    }
    p.fits = n <= LIST;
    return p;
}

template <typename T>
__global__ void __launch_bounds__(CT) chunk_list_kernel(const CutArgs a, RowState* __restrict__ st, int chunk, bool vec) {
    __shared__ CutLds<CT> l;
    const int row = blockIdx.y, tid = threadIdx.x;
    const Setting s = setting_of(a.how, row);
    RowState& r = st[row];
    const float m = row_max(r, gridDim.x);
    if (!s.ok || !(m > -INFINITY)) return;
    const Plan pl = plan_of<CT>(l, r, s);
    const T* p = (const T*)a.logits + (size_t)row * a.ld;
    const int lo = blockIdx.x * chunk, hi = min(a.vocab, lo + chunk);
    uint64_t sum = 0;
    unsigned n = 0;
    for_chunk(p, lo, hi, vec, [&](float x, int i) {
        const float z = __fmul_rn(x, s.inv);
        const uint64_t w = score_weight(z, m);
        if (!w) return;
        const int b = bin_of(dist_bits(z, m));
        if (b < pl.lo) {
            if (w >= s.least) {
                sum += w;
                ++n;
            }
        } else if (pl.fits && (b <= pl.hi || (pl.listed_k && b == pl.k.bin))) {
            const unsigned at = atomicAdd(&r.listed, 1u);
            r.list[at].z = z;
            r.list[at].idx = i;
        }
    });
    sum = block_reduce<CT>(l, sum, [](uint64_t x, uint64_t y) { return x + y; });
    n = block_reduce<CT>(l, n, [](unsigned x, unsigned y) { return x + y; });
    if (tid == 0) {
        r.chunk_mass[blockIdx.x] = sum;
        r.chunk_cnt[blockIdx.x] = n;
    }
}

constexpr int FT = 1024;
template <typename T>
__global__ void __launch_bounds__(FT) row_end_kernel(const CutArgs a, RowState* __restrict__ st, int chunk, int chunks, bool vec) {
    __shared__ CutLds<FT> l;
    __shared__ float lz[LIST];
    __shared__ unsigned li[LIST];
    __shared__ unsigned long long cm[CHUNKS];
    __shared__ unsigned s_kept;
    const int row = blockIdx.x, tid = threadIdx.x, vocab = a.vocab;
    const Setting s = setting_of(a.how, row);
    RowState& r = st[row];
    const T* p = (const T*)a.logits + (size_t)row * a.ld;
    const float m = row_max(r, chunks);
    RowCut c = uncut(s, m);
    if (!s.ok || !(m > -INFINITY)) {
        if (tid == 0) {
            if (a.cut) a.cut[row] = c;
            if (a.u) emit(a, row, -1, 0, 0, 0);
        }
        return;
    }
    const Plan pl = plan_of<FT>(l, r, s);
    const int n = pl.fits && pl.lo < BINS ? (int)r.listed : 0;
    for (int i = tid; i < n; i += FT) {
        lz[i] = r.list[i].z;
        li[i] = r.list[i].idx;
    }
    if (tid < CHUNKS) cm[tid] = tid < chunks ? r.chunk_mass[tid] : 0;
    if (tid == 0) s_kept = 0;
    __syncthreads();
    auto each = [&](auto&& fn) {
        if (pl.fits)
            for (int i = tid; i < n; i += FT) fn(lz[i], li[i]);
        else
            for (int i = tid; i < vocab; i += FT) fn(__fmul_rn(logit(p, i), s.inv), (unsigned)i);
    };
    if (pl.lo < BINS) cut_along<FT>(l, r.mass, r.cnt, s, each, c);
    // what the cut leaves of the listed bins joins what the chunks have for sure
    unsigned kept = tid < chunks ? r.chunk_cnt[tid] : 0;
    if (pl.lo < BINS)
        each([&](float z, unsigned i) {
            const uint64_t w = cut_weight(c, z, i);
            if (!w || bin_of(dist_bits(z, m)) < pl.lo) return;
            atomicAdd(&cm[i / chunk], (unsigned long long)w);
            ++kept;
        });
    if (kept) atomicAdd(&s_kept, kept);
    __syncthreads();
    uint64_t R = 0;
    for (int k = 0; k < chunks; ++k) R += cm[k];
    c.R = R;
    if (a.cut && tid == 0) a.cut[row] = c;
    if (!a.u) return;
    const uint64_t target = draw_target(a, row, R);
    uint64_t base = 0;
    int at = 0;
    while (at + 1 < chunks && base + cm[at] <= target) base += cm[at++];
    const int lo = at * chunk, hi = min(vocab, lo + chunk);
    for (int i0 = lo; i0 < hi; i0 += FT * 4) {
        const int i = i0 + tid * 4;
        f32x4 x{NAN, NAN, NAN, NAN};
        if (vec && i + 4 <= hi) x = logits4(p + i);
        else
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (i + e < hi) x[e] = logit(p, i + e);
        uint64_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = cut_weight(c, __fmul_rn(x[e], s.inv), i + e);
        const int f = first_over<FT>(l, w, base, target);
        if (f < 0) continue;
        if (f / 4 == tid) emit(a, row, i0 + f, f % 4 == 0 ? w[0] : f % 4 == 1 ? w[1] : f % 4 == 2 ? w[2] : w[3], R, s_kept);
        return;
    }
}

constexpr int ROW_MOST = 8192;  // longest row that one workgroup takes alone

int row_chunks(int rows, int vocab) { return std::max(1, std::min(std::min(CHUNKS, (vocab + 2047) / 2048), std::max(512 / rows, (vocab + 16383) / 16384))); }

template <typename T>
hipError_t launch(const CutArgs& a, void* work, hipStream_t s) {
    const bool vec = a.ld % 4 == 0 && ((uintptr_t)a.logits & (4 * sizeof(T) - 1)) == 0;
    if (a.vocab <= ROW_MOST) {
        const dim3 g(a.rows);
        if (a.vocab <= 2048) hipLaunchKernelGGL((cut_row_kernel<T, 256, 2048>), g, dim3(256), 0, s, a, vec);
        else hipLaunchKernelGGL((cut_row_kernel<T, 1024, ROW_MOST>), g, dim3(1024), 0, s, a, vec);
        return hipGetLastError();
    }
    RowState* st = (RowState*)work;
    int chunks = row_chunks(a.rows, a.vocab);
    const int chunk = ((a.vocab + chunks - 1) / chunks + 3) & ~3;
    chunks = (a.vocab + chunk - 1) / chunk;
    const dim3 g(chunks, a.rows);
    hipLaunchKernelGGL(chunk_max_kernel<T>, g, dim3(CT), 0, s, a, st, chunk, vec);
    hipLaunchKernelGGL(chunk_bins_kernel<T>, g, dim3(CT), 0, s, a, st, chunk, vec);
    hipLaunchKernelGGL(chunk_list_kernel<T>, g, dim3(CT), 0, s, a, st, chunk, vec);
    hipLaunchKernelGGL(row_end_kernel<T>, dim3(a.rows), dim3(FT), 0, s, a, st, chunk, chunks, vec);
    return hipGetLastError();
}

}  // namespace

size_t cut_workspace_bytes(int rows, int vocab) { return vocab <= ROW_MOST ? 256 : (size_t)rows * sizeof(RowState); }

hipError_t launch_cut(int dtype, const CutArgs& a, void* work, hipStream_t s) { return dtype == 0 ? launch<float>(a, work, s) : launch<bf16_t>(a, work, s); }
