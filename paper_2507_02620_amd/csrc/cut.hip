// Sampling of a token per row under temperature, top-k, top-p and min-p, and the same cuts for acceptance along a tree.
//
// Scores z = logit * (1 / temperature) are rounded once to 32 bits; weights are the whole numbers of exp_weight, so sums have no order and
// every comparison is exact.  Order of a row: z descending, index ascending.  top-k keeps its first k; S is their sum; top-p keeps the
// shortest part whose sum reaches ceil(P S / 2^30), P = floor(p 2^30); min-p what weighs at least ceil(min_p 2^32).  The token is the first kept
// one by index whose running sum exceeds floor(U R / 2^48), R the sum of what is kept, U = floor(u 2^48).
//
// Nothing is sorted: a row's scores are counted and weighed in bins along the order, a scan finds the bin in which a cut falls, and only that bin's scores are
// looked at more closely, by digits of their distance, score and index.  Counts and weights are whole numbers, so the order of the atomics changes nothing.
//
// Bound: the rows are read once under top-k, else three times, from the caches after the first (64 rows x 152064 in 32 bits, 39 MB, floor 7.6 us); what takes the
// time are LDS atomics, scans and barriers one after the other: 10.2 us for the maxima, 11.6 bins, 12.9 lists, 22.2 the rows' ends, of which every one is a
// chain of 6 to 12 dependent steps.  Short rows: latency and the call (1024 scores 5.7 us).  One launch with a row to a workgroup took 1190 us for those 64 rows.
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

// ---- a wave's sums by lane moves (a shuffle goes through the LDS) ----
template <int CTRL, int ROWS>
static __device__ __forceinline__ unsigned moved(unsigned v, unsigned none) {
    return (unsigned)__builtin_amdgcn_update_dpp((int)none, (int)v, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS>
static __device__ __forceinline__ uint64_t moved(uint64_t v, uint64_t) {
    return (uint64_t)moved<CTRL, ROWS>((unsigned)(v >> 32), 0u) << 32 | moved<CTRL, ROWS>((unsigned)v, 0u);
}
template <int CTRL, int ROWS>
static __device__ __forceinline__ float moved(float v, float none) {
    return __uint_as_float(moved<CTRL, ROWS>(__float_as_uint(v), __float_as_uint(none)));
}
struct Sum {
    template <typename V>
    __device__ __forceinline__ V operator()(V x, V y) const { return x + y; }
};
struct Max {
    __device__ __forceinline__ float operator()(float x, float y) const { return fmaxf(x, y); }
};
// f over the lanes up to and with this one: shifts by 1, 2, 4, 8 in rows of 16 lanes, then the rows' last lanes into the rows behind them.
template <typename V, typename F>
static __device__ __forceinline__ V wave_upto(V v, V none, F f) {
    v = f(v, moved<0x111, 0xf>(v, none));
    v = f(v, moved<0x112, 0xf>(v, none));
    v = f(v, moved<0x114, 0xf>(v, none));
    v = f(v, moved<0x118, 0xf>(v, none));
    v = f(v, moved<0x142, 0xa>(v, none));
    return f(v, moved<0x143, 0xc>(v, none));
}
static __device__ __forceinline__ unsigned of_lane(unsigned v, int j) { return (unsigned)__builtin_amdgcn_readlane((int)v, j); }
static __device__ __forceinline__ uint64_t of_lane(uint64_t v, int j) { return (uint64_t)of_lane((unsigned)(v >> 32), j) << 32 | of_lane((unsigned)v, j); }
static __device__ __forceinline__ float of_lane(float v, int j) { return __uint_as_float(of_lane(__float_as_uint(v), j)); }
template <typename V, typename F>
static __device__ __forceinline__ V wave_all(V v, V none, F f) { return of_lane(wave_upto(v, none, f), 63); }

// ---- bins: scores by their distance from the row's largest ---------------------------------------------------------------------
// 32 bins to a power of two of the distance d = fl(m - z), from 2^-20 on; bin 0 is what lies nearer.  d falls as z rises, so bins keep the order.
// Weights end at d = 32 ln 2 = 22.2; what lies behind DMAX counts nowhere.  Relative bins suit every scale of scores: of N(0, s^2) rows the fullest
// one holds 5 % whatever s.
constexpr unsigned D0 = 0x35800000u, DMAX = 0x41b20000u;  // 2^-20, 22.25
constexpr int BIN_SHIFT = 18, BINS = 800;
static_assert(((DMAX - D0) >> BIN_SHIFT) + 1 < BINS, "every distance below DMAX has a bin");
static __device__ __forceinline__ unsigned dist_bits(float z, float m) { return z == m ? 0u : __float_as_uint(sub_once(m, z)); }
static __device__ __forceinline__ int bin_of(unsigned d) { return d < D0 ? 0 : (int)((d - D0) >> BIN_SHIFT) + 1; }

// ---- selection -------------------------------------------------------------------------------------------------------------------
constexpr int DIGIT = 10, FEW = 64;
struct Tally {  // of bins
    unsigned long long mass[BINS];
    unsigned cnt[BINS];
};
struct Found {
    int bin;               // the first one with which the running count, or weight, reaches the need; -1: none does, and the sums are those of all
    unsigned cnt, in_cnt;  // before it; in it
    uint64_t mass, in_mass;
};
struct Bound {  // the last element that is kept
    float z;
    unsigned idx;
    unsigned cnt;  // up to and with it
    uint64_t mass;
};
// Digits lie a place further apart after every 16, which are a lane's: without it all lanes read from two banks.
constexpr int DIGITS = (1 << DIGIT) + (1 << DIGIT) / 16;
static __device__ __forceinline__ int digit_at(int d) { return d + (d >> 4); }
template <int NT>
struct CutLds {
    unsigned long long mass[DIGITS];
    unsigned cnt[DIGITS];
    unsigned long long red[NT / 64];
    Bound bound;
    float fz[FEW];
    unsigned fi[FEW], fn, zmin, zmax;
};
static __device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// N counts and weights in order, N / 64 to a lane, and what comes before a lane's: looked up as often as needed, by one look at the lane's own and one at
// its entries.  Every wave does so by itself, without a barrier.
template <int N>
struct Scan {
    static constexpr int E = (N + 63) / 64;
    static_assert(E <= 16, "a lane's entries fit a row of lanes");
    const unsigned long long* mass;
    const unsigned* cnt;
    int n;
    unsigned c, cb, ct;
    uint64_t m, mb, mt;
    static __device__ __forceinline__ int place(int i) { return N == 1 << DIGIT ? digit_at(i) : i; }
    __device__ __forceinline__ void make(const unsigned long long* mass_, const unsigned* cnt_, int n_, unsigned cnt0, uint64_t mass0) {
        mass = mass_;
        cnt = cnt_;
        n = n_;
        const int first = (threadIdx.x & 63) * E;
        c = 0;
        m = 0;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            c += first + i < n ? cnt[place(first + i)] : 0;
            m += first + i < n ? mass[place(first + i)] : 0;
        }
        const unsigned cu = wave_upto(c, 0u, Sum{});
        const uint64_t mu = wave_upto(m, (uint64_t)0, Sum{});
        cb = cnt0 + cu - c;
        mb = mass0 + mu - m;
        ct = cnt0 + of_lane(cu, 63);
        mt = mass0 + of_lane(mu, 63);
    }
    __device__ __forceinline__ Found find(uint64_t need, bool by_count) const {
        if ((by_count ? ct : mt) < need) return Found{-1, ct, 0, mt, 0};
        const int lane = threadIdx.x & 63;
        const unsigned long long reach = __ballot(by_count ? cb + c >= need : mb + m >= need);
        const int from = (__ffsll(reach) - 1) * E, i = from + lane;
        const bool mine = lane < E && i < n;
        const unsigned x = mine ? cnt[place(i)] : 0;
        const uint64_t y = mine ? mass[place(i)] : 0;
        unsigned xs = x;
        uint64_t ys = y;
        xs += moved<0x111, 0xf>(xs, 0u);
        ys += moved<0x111, 0xf>(ys, (uint64_t)0);
        xs += moved<0x112, 0xf>(xs, 0u);
        ys += moved<0x112, 0xf>(ys, (uint64_t)0);
        xs += moved<0x114, 0xf>(xs, 0u);
        ys += moved<0x114, 0xf>(ys, (uint64_t)0);
        xs += moved<0x118, 0xf>(xs, 0u) + of_lane(cb, from / E);
        ys += moved<0x118, 0xf>(ys, (uint64_t)0) + of_lane(mb, from / E);
        const int at = __ffsll(__ballot(mine && (by_count ? xs >= need : ys >= need))) - 1;
        const unsigned in = of_lane(x, at);
        const uint64_t win = of_lane(y, at);
        return Found{from + at, of_lane(xs, at) - in, in, of_lane(ys, at) - win, win};
    }
};

// The last kept element of bin f.bin: the one at which the running count (or weight) along the order, `f` before the bin, first reaches the need.
// Digits of ten bits of d, then of z's key, then of the index, until a wave can rank what is left.  each(fn) calls fn(z, index) for
// the elements of the row, or at least for all of that bin, in any order.
template <int NT, typename L, typename Each>
static __device__ __forceinline__ Bound select_in(L& l, float m, Found f, uint64_t need, bool by_count, const Each& each) {
    const int tid = threadIdx.x, bin = f.bin;
    unsigned d_at = bin ? (D0 >> BIN_SHIFT) + bin - 1 : 0, z_at = 0, i_at = 0;  // digits found so far
    int d_sh = bin ? BIN_SHIFT : 30, z_sh = 32, i_sh = 20;
    auto member = [&](float z, unsigned i, unsigned& d, unsigned& k) {
        d = dist_bits(z, m);
        k = down_key(z);
        if ((uint64_t)d >> d_sh != d_at || d >= (bin ? DMAX : D0)) return false;
        return d_sh > 0 || ((uint64_t)k >> z_sh == z_at && (z_sh > 0 || i >> i_sh == i_at));
    };
    while (f.in_cnt > FEW) {
        if (d_sh == 0 && z_sh == 32) {  // the same distance: mostly the same score
            __syncthreads();
            if (tid == 0) {
                l.zmin = ~0u;
                l.zmax = 0u;
            }
            __syncthreads();
            each([&](float z, unsigned i) {
                unsigned d, k;
                if (member(z, i, d, k)) {
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
        for (int i = tid; i < n + n / 16; i += NT) {
            l.mass[i] = 0;
            l.cnt[i] = 0;
        }
        __syncthreads();
        each([&](float z, unsigned i) {
            unsigned d, k;
            if (!member(z, i, d, k)) return;
            const int at = digit_at(((level == 0 ? d : level == 1 ? k : i) >> to) & (n - 1));
            atomicAdd(&l.cnt[at], 1u);
            atomicAdd(&l.mass[at], (unsigned long long)score_weight(z, m));
        });
        __syncthreads();
        Scan<1 << DIGIT> scan;
        scan.make(l.mass, l.cnt, n, f.cnt, f.mass);
        f = scan.find(need, by_count);
        unsigned& at = level == 0 ? d_at : level == 1 ? z_at : i_at;
        at = at << (from - to) | f.bin;
        (level == 0 ? d_sh : level == 1 ? z_sh : i_sh) = to;
    }
    __syncthreads();
    if (tid == 0) l.fn = 0;
    __syncthreads();
    each([&](float z, unsigned i) {
        unsigned d, k;
        if (!member(z, i, d, k)) return;
        const unsigned at = atomicAdd(&l.fn, 1u);
        l.fz[at] = z;
        l.fi[at] = i;
    });
    __syncthreads();
    if (tid < 64) {
        const int n = uniform((int)l.fn);
        const float z = tid < n ? l.fz[tid] : NAN;
        const unsigned i = tid < n ? l.fi[tid] : 0;
        const uint64_t w = tid < n ? score_weight(z, m) : 0;
        unsigned c = f.cnt;
        uint64_t s = f.mass;
        for (int j = 0; j < n; ++j) {
            const float zj = of_lane(z, j);
            const unsigned ij = of_lane(i, j);
            const uint64_t wj = of_lane(w, j);
            if (zj > z || (zj == z && ij < i)) {
                ++c;
                s += wj;
            }
        }
        if (tid < n && (by_count ? c + 1 == need : s < need && s + w >= need)) l.bound = Bound{z, i, c + 1, s + w};
    }
    __syncthreads();
    return l.bound;
}

// The element at which the running weight along the index first exceeds `target`, of those that each(fn) gives with fn(weight, index).
template <int NT, typename L, typename Each>
static __device__ __forceinline__ Bound select_index(L& l, uint64_t target, unsigned n_all, const Each& each) {
    const int tid = threadIdx.x;
    Found f{0, 0, n_all, 0, 0};
    unsigned at = 0;
    int sh = 20;
    while (sh > 0 && f.in_cnt > FEW) {
        const int to = max(sh - DIGIT, 0), n = 1 << (sh - to);
        __syncthreads();
        for (int i = tid; i < n + n / 16; i += NT) {
            l.mass[i] = 0;
            l.cnt[i] = 0;
        }
        __syncthreads();
        each([&](uint64_t w, unsigned i) {
            if (i >> sh != at) return;
            atomicAdd(&l.cnt[digit_at((i >> to) & (n - 1))], 1u);
            atomicAdd(&l.mass[digit_at((i >> to) & (n - 1))], (unsigned long long)w);
        });
        __syncthreads();
        Scan<1 << DIGIT> scan;
        scan.make(l.mass, l.cnt, n, 0, f.mass);
        f = scan.find(target + 1, false);
        at = at << (sh - to) | f.bin;
        sh = to;
    }
    __syncthreads();
    if (tid == 0) l.fn = 0;
    __syncthreads();
    each([&](uint64_t w, unsigned i) {
        if (i >> sh != at) return;
        const unsigned k = atomicAdd(&l.fn, 1u);
        l.mass[k] = w;
        l.fi[k] = i;
    });
    __syncthreads();
    if (tid < 64) {
        const int n = uniform((int)l.fn);
        const unsigned i = tid < n ? l.fi[tid] : 0;
        const uint64_t w = tid < n ? l.mass[tid] : 0;
        uint64_t s = f.mass;
        for (int j = 0; j < n; ++j) {
            const unsigned ij = of_lane(i, j);
            const uint64_t wj = of_lane(w, j);
            s += ij < i ? wj : 0;
        }
        if (tid < n && s <= target && target < s + w) l.bound = Bound{0.f, i, 0, w};
    }
    __syncthreads();
    return l.bound;
}

template <int NT, typename V, typename L, typename F>
static __device__ __forceinline__ V block_reduce(L& l, V v, V none, F f) {  // ends with a barrier
    V* sh = (V*)l.red;
    v = wave_all(v, none, f);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    v = sh[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) v = f(v, sh[w]);
    __syncthreads();
    return v;
}

// (a row without a score above -inf keeps nothing: no z is above its bound)
static __device__ __forceinline__ RowCut uncut(const Setting& s, float m) {
    return RowCut{m, m > -INFINITY && s.ok ? -INFINITY : INFINITY, ~0u, (unsigned)s.least, (unsigned)(s.least >> 32), 0, 0};
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

// The whole of a row whose top-k lies among n <= 64 scores, in l.fz and l.fi: the waves rank them, along the order and along the index, by comparing all of
// them with a share each; then the first wave sums in order, by lane moves, and draws.
template <int NT, typename L>
static __device__ __forceinline__ void few_end(L& l, const CutArgs& a, int row, const Setting& s, RowCut& c) {
    constexpr int W = NT / 64;
    const int lane = threadIdx.x & 63, wv = uniform(threadIdx.x >> 6), n = uniform((int)l.fn);
    const float z = lane < n ? l.fz[lane] : NAN;
    const unsigned i = lane < n ? l.fi[lane] : ~0u;
    const uint64_t key = (uint64_t)down_key(z) << 32 | i;
    unsigned ranks = 0;  // along the order below, along the index above
    for (int j = wv; j < n; j += W) {
        const uint64_t kj = of_lane(key, j);
        ranks += (kj < key ? 1u : 0u) + ((unsigned)kj < i ? 1u << 16 : 0u);
    }
    l.cnt[threadIdx.x] = ranks;
    __syncthreads();
    if (wv) return;
    ranks = 0;
#pragma unroll
    for (int k = 0; k < W; ++k) ranks += l.cnt[k * 64 + lane];
    // (one wave's own stores and loads, in order; places from 64 on: the sorted scores, weights, ranks; then kept weights and indexes by index)
    const int at = lane < n ? (int)(ranks & 0xffff) : lane, at_i = lane < n ? (int)(ranks >> 16) : lane;
    l.mass[64 + at] = lane < n ? score_weight(z, c.m) : 0;
    l.cnt[64 + at] = (unsigned)at_i;
    l.cnt[128 + at_i] = i;
    l.fz[at] = z;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const uint64_t w = l.mass[64 + lane], upto = wave_upto(w, (uint64_t)0, Sum{});
    const int first = min((int)min(s.k, 64u), n);
    bool keep = lane < first;
    if (s.P < (1u << 30)) keep &= upto - w < top_p_need(s.P, of_lane(upto, first - 1));
    const int last = __popcll(__ballot(keep)) - 1;  // along the order
    const uint64_t mine = keep && w >= s.least ? w : 0;
    const unsigned kept = __popcll(__ballot(mine != 0)), my_i = l.cnt[64 + lane];
    l.mass[128 + my_i] = mine;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const uint64_t wi = l.mass[128 + lane], run = wave_upto(wi, (uint64_t)0, Sum{}), R = of_lane(run, 63);
    if (a.cut && lane == last) {
        c.z = l.fz[lane];
        c.idx = l.cnt[128 + my_i];
        c.R = R;
        a.cut[row] = c;
    }
    if (!a.u) return;
    const uint64_t target = draw_target(a, row, R);
    if (run > target && run - wi <= target) emit(a, row, (int)l.cnt[128 + lane], wi, R, kept);
}

// What top-k, then top-p over what that leaves, keep of a row whose bins t are.
// `whole`: each(fn) gives all of the row's first bins, and under top-k the bins hold no weights yet.  Returns true where that was all: the row's cut and token are out.
template <int NT, typename L, typename Each>
static __device__ __forceinline__ bool cut_along(L& l, Tally& t, const CutArgs& a, int row, const Setting& s, bool whole, const Each& each, RowCut& c) {
    __syncthreads();
    Scan<BINS> scan;
    scan.make(t.mass, t.cnt, BINS, 0, 0);
    uint64_t need = s.k;
    bool by_count = s.k != 0;
    if (!by_count) need = top_p_need(s.P, scan.mt);
#pragma nounroll
    for (;;) {  // once or twice
        Found f = scan.find(need, by_count);
        if (whole && by_count) {
            const int last = f.bin < 0 ? BINS : f.bin;
            if (f.cnt + f.in_cnt > FEW) {  // weights of what top-k can keep
                each([&](float z, unsigned) {
                    const unsigned d = dist_bits(z, c.m);
                    if (d < DMAX && bin_of(d) <= last) atomicAdd(&t.mass[bin_of(d)], (unsigned long long)score_weight(z, c.m));
                });
                __syncthreads();
                scan.make(t.mass, t.cnt, BINS, 0, 0);
                f = scan.find(need, true);
            } else {
                if (threadIdx.x == 0) l.fn = 0;
                __syncthreads();
                each([&](float z, unsigned i) {
                    const unsigned d = dist_bits(z, c.m);
                    if (d >= DMAX || bin_of(d) > last) return;
                    const unsigned at = atomicAdd(&l.fn, 1u);
                    l.fz[at] = z;
                    l.fi[at] = i;
                });
                __syncthreads();
                few_end<NT>(l, a, row, s, c);
                return true;
            }
        }
        uint64_t S = scan.mt;
        if (f.bin >= 0) {
            const Bound b = select_in<NT>(l, c.m, f, need, by_count, each);
            c.z = b.z;
            c.idx = b.idx;
            S = b.mass;
        }
        if (!by_count || s.P >= (1u << 30)) return false;
        need = top_p_need(s.P, S);
        by_count = false;
    }
}

static __device__ __forceinline__ void count_in(Tally& t, float z, float m) {
    const unsigned d = dist_bits(z, m);
    if (d >= DMAX) return;
    atomicAdd(&t.cnt[bin_of(d)], 1u);
    atomicAdd(&t.mass[bin_of(d)], (unsigned long long)score_weight(z, m));
}

// The first of the block's NT * 4 consecutive entries (four of a thread's, w their weights) with which the running sum, `base` before them, exceeds
// the target; -1 if none does.  base becomes the sum behind them.  Two barriers.
template <int NT, typename L>
static __device__ __forceinline__ int first_over(L& l, const uint64_t (&w)[4], uint64_t& base, uint64_t target) {
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const uint64_t own = w[0] + w[1] + w[2] + w[3];
    const uint64_t run = wave_upto(own, (uint64_t)0, Sum{});
    __syncthreads();
    if (lane == 63) l.red[wv] = run;
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
        l.fi[0] = tid * 4 + e;
    }
    __syncthreads();
    return (int)l.fi[0];
}

// ---- a row per workgroup, its scores in LDS: one launch ----------------------------------------------------------------------
// (up to 8192 scores, us a call, against rows in chunks: 16 rows x 6000 top-p 18.2, 30.3; 16 x 8000 top-k 50 8.9, 12.5; 200 x 8000 top-p 20.4, 34.3)
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
            x[e] = mul_once(x[e], s.inv);
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
    m = block_reduce<NT>(l, m, -INFINITY, Max{});
    RowCut c = uncut(s, m);
    const bool any = s.ok && m > -INFINITY;
    auto each = [&](auto&& fn) __attribute__((always_inline)) {
        for (int i = tid * 4; i < vocab; i += NT * 4) {
            const f32x4 x = *(const f32x4*)(z + i);
#pragma unroll
            for (int e = 0; e < 4; ++e) fn(x[e], (unsigned)(i + e));  // (what lies behind the row weighs nothing)
        }
    };
    if (any && along) {
        if (s.k)
            each([&](float x, unsigned) {
                const unsigned d = dist_bits(x, m);
                if (d < DMAX) atomicAdd(&t.cnt[bin_of(d)], 1u);
            });
        else
            each([&](float x, unsigned) { count_in(t, x, m); });
        if (cut_along<NT>(l, t, a, row, s, true, each, c)) return;
    }
    unsigned kept = 0;
    uint64_t R = 0;
    if (any) {
        each([&](float x, unsigned i) {
            const uint64_t w = cut_weight(c, x, i);
            R += w;
            kept += w != 0;
        });
        R = block_reduce<NT>(l, R, (uint64_t)0, Sum{});
    }
    c.R = R;
    if (a.cut && tid == 0) a.cut[row] = c;
    if (!a.u) return;
    if (!any) {
        if (tid == 0) emit(a, row, -1, 0, 0, 0);
        return;
    }
    kept = block_reduce<NT>(l, kept, 0u, Sum{});
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
// A row under top-k is settled by its chunks' own top-k: one pass, in which a chunk lists every score that can be among the row's first k, and a workgroup
// per row over the lists.  Other rows need the row's largest score first and all weights then: the chunks' maxima; the chunks' bins, which add up to the
// row's; the scores of the bins that the cuts pass through, to a list; and a workgroup per row that finds the cut in the list and the token in
// the chunk that the target falls into.  (One compute unit alone would take 25 us to look through a row of 152064 in memory.)
constexpr int CHUNKS = 256, LIST = 16384, CT = 256, CHUNK_LEAST = CT * 4 * 4, CHUNK_MOST = CT * 4 * 12, STAGE = 1024;
static_assert((long long)CHUNKS * CHUNK_LEAST >= CUT_MAX_VOCAB, "the longest row has a place");
constexpr unsigned OVER = ~0u;
struct Entry {
    float z;
    unsigned idx;
};
// Weights and counts meet in one word: a chunk's weights sum to less than 2^47, its entries are fewer than 2^16.
constexpr int PACK = 48;
constexpr unsigned long long LOW = (1ull << PACK) - 1;
static_assert(CHUNK_MOST < 1 << (64 - PACK) && CHUNK_MOST <= 1 << (PACK - 33), "no sum leaves its half");
// Which bins of a row that its chunks do not settle hold its cuts: [lo, hi], and k; below lo everything is kept, behind hi nothing, but that top-k's end
// needs its own bin looked at.
struct Plan {
    int lo, hi, k;  // k: -1 if none
    bool order;     // a cut along the order counts
    bool fits;      // the list holds them
};
struct alignas(16) RowState {
    Tally t;                          // of the row
    unsigned own[CHUNKS];             // entries of a chunk's part of the list (rows under top-k); OVER: more than fit
    float max[CHUNKS];
    unsigned long long sure[CHUNKS];  // what of a chunk is kept whatever the listed bins' share is: count and weight
    Plan plan;                        // of rows that their chunks do not settle
    unsigned listed;                  // entries of the list (rows that their chunks do not settle)
    Entry list[LIST];
    __device__ __forceinline__ unsigned long long* bins(int c) { return (unsigned long long*)(this + 1) + (size_t)c * BINS; }  // [chunks][BINS] behind it
};
static_assert(sizeof(RowState) % 16 == 0, "what is behind it is aligned");
size_t row_bytes(int chunks) { return sizeof(RowState) + (size_t)chunks * BINS * 8; }
struct ChunkArgs {
    char* state;  // [rows] of `stride` bytes
    size_t stride;
    int chunk, chunks;
    bool vec;    // rows on 16 bytes (8 of 16-bit logits)
    bool later;  // the launches for rows that are not settled by their chunks follow
    __device__ __forceinline__ RowState& row(int i) const { return *(RowState*)(state + stride * i); }
};
// Entries of a chunk's part of the list.
static __host__ __device__ __forceinline__ int own_most(int chunks) { return LIST / chunks; }
// Rows under a larger top-k are not settled by their chunks, as a list that overflows sends its row back to memory: 64 rows x 152064, 38 lists, us a call:
// top-k 200 37.7 by lists; 300 43.8 by lists, 58.6 the other way; 400 245 by lists, some of which overflow, 60.2 the other way.
// Where many scores are equal or nearly so, lists overflow under any top-k and under top-p, and a workgroup goes through its row in memory, with all lanes'
// atomics in one bin.  64 rows x 152064, us a call, scores of N(0, 4), the same as multiples of 1/2, all equal: top-k 50 20.6, 36.4, 2707; with top-p 0.9 besides
// 20.8, 39.8, 5090; top-p 0.9 64.9, 237, 2567; one row of equal scores among the 64 takes as long.  (Lanes that meet in a bin with one weight added up before: all
// equal 877, 1574, 890, but 16 rows x 8000 under top-p 19.0 -> 24.0.)  A row of 2^20 scores fills a list by itself: N(0, 4) under top-p 1.2 ms.
static __host__ __device__ __forceinline__ int top_most(int chunks) { return LIST / 2 / chunks; }
static __device__ __forceinline__ bool by_chunks(const Setting& s, const ChunkArgs& ch) { return s.k && s.k <= (unsigned)top_most(ch.chunks); }

// A thread's scores of a chunk: score (j * CT + tid) * 4 + e of it; what lies behind its end weighs nothing.  (No branch around a load; where rows lie on
// 16 bytes, chunks end there too.)
template <typename T, int NV>
static __device__ __forceinline__ void load_chunk(f32x4 (&x)[NV], const T* p, int lo, int hi, bool vec, float inv) {
    const int i0 = lo + (int)threadIdx.x * 4;
    if (vec) {
#pragma unroll
        for (int j = 0; j < NV; ++j) x[j] = logits4(p + min(i0 + j * CT * 4, hi - 4));
    } else {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[j][e] = logit(p, min(i0 + j * CT * 4 + e, hi - 1));
    }
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[j][e] = i0 + j * CT * 4 + e < hi ? mul_once(x[j][e], inv) : NAN;
}

template <typename T, int NV>
__global__ void __launch_bounds__(CT, 4) chunk_top_kernel(const CutArgs a, const ChunkArgs ch) {
    __shared__ struct {
        unsigned long long red[CT / 64];
        unsigned fn;
        int last;
    } l;
    __shared__ unsigned cnt[BINS];
    const int row = blockIdx.y, c = blockIdx.x, tid = threadIdx.x;
    RowState& r = ch.row(row);
    const int lo = c * ch.chunk, hi = min(a.vocab, lo + ch.chunk), n = hi - lo;
    const Setting s = setting_of(a.how, row);
    f32x4 z[NV];
    load_chunk<T, NV>(z, (const T*)a.logits + (size_t)row * a.ld, lo, hi, ch.vec, s.inv);
    if (ch.later) {  // for the launches behind this one
        for (int i = c * CT + tid; i < BINS; i += ch.chunks * CT) {
            r.t.mass[i] = 0;
            r.t.cnt[i] = 0;
        }
        if (c == 0 && tid == 0) r.listed = 0;
    }
    const bool top = by_chunks(s, ch);
    if (top)
        for (int i = tid; i < BINS; i += CT) cnt[i] = 0;
    if (tid == 0) l.fn = 0;
    float m = -INFINITY, m4[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        m4[j] = fmaxf(fmaxf(z[j][0], z[j][1]), fmaxf(z[j][2], z[j][3]));
        m = fmaxf(m, m4[j]);
    }
    const float mine = m;
    m = block_reduce<CT>(l, m, -INFINITY, Max{});
    if (tid == 0) r.max[c] = m;
    if (!top) return;
    if (m == -INFINITY) {
        if (tid == 0) r.own[c] = 0;
        return;
    }
    // The k-th largest of the maxima of groups is no larger than the k-th largest score: where the groups' count reaches k, so does the scores'.  A group is a
    // thread's scores, or four of them where k is large (64 rows x 152064, of which half under top-k: 10.2 us, counting every score 20).
    auto count = [&](float x) {
        const unsigned d = dist_bits(x, m);
        if (d < DMAX) atomicAdd(&cnt[bin_of(d)], 1u);
    };
    if (s.k <= CT / 2) {
        count(mine);
    } else {
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (j * CT * 4 < n) count(m4[j]);
    }
    __syncthreads();
    if (tid < 64) {
        constexpr int E = (BINS + 63) / 64;
        unsigned own[E], sum = 0;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            own[i] = tid * E + i < BINS ? cnt[tid * E + i] : 0;
            sum += own[i];
        }
        unsigned before = wave_upto(sum, 0u, Sum{}) - sum;
        int at = BINS;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            before += own[i];
            at = at == BINS && before >= s.k ? tid * E + i : at;
        }
        const unsigned long long reach = __ballot(at < BINS);
        if (tid == 0) l.last = reach ? (int)of_lane((unsigned)at, __ffsll(reach) - 1) : BINS;
    }
    __syncthreads();
    const int last = uniform(l.last);
    const unsigned most = (unsigned)own_most(ch.chunks);
    Entry* to = r.list + c * most;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const unsigned d4 = dist_bits(m4[j], m);
        if (j * CT * 4 < n && d4 < DMAX && bin_of(d4) <= last)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const unsigned d = dist_bits(z[j][e], m);
                if (d < DMAX && bin_of(d) <= last) {
                    const unsigned at = atomicAdd(&l.fn, 1u);
                    if (at < most) to[at] = Entry{z[j][e], (unsigned)(lo + (j * CT + tid) * 4 + e)};
                }
            }
    }
    __syncthreads();
    if (tid == 0) r.own[c] = l.fn > most ? OVER : l.fn;
}

// The row's largest score, and whether its chunks settled it (every wave by itself).
static __device__ __forceinline__ float row_max(const RowState& r, int chunks, bool top, bool& settled) {
    float m = -INFINITY;
    bool ok = top;
    for (int i = threadIdx.x & 63; i < chunks; i += 64) {
        m = fmaxf(m, r.max[i]);
        if (top) ok &= r.own[i] != OVER;
    }
    settled = __ballot(!ok) == 0;
    return wave_all(m, -INFINITY, Max{});
}

template <typename T, int NV>
__global__ void __launch_bounds__(CT, 4) chunk_bins_kernel(const CutArgs a, const ChunkArgs ch) {
    __shared__ unsigned long long t[BINS];
    __shared__ struct {
        unsigned long long red[CT / 64];
    } l;
    const int row = blockIdx.y, tid = threadIdx.x;
    const Setting s = setting_of(a.how, row);
    RowState& r = ch.row(row);
    bool settled;
    const float m = row_max(r, ch.chunks, by_chunks(s, ch), settled);
    if (settled || !s.ok || !(m > -INFINITY)) return;
    const int lo = blockIdx.x * ch.chunk, hi = min(a.vocab, lo + ch.chunk), n = hi - lo;
    f32x4 z[NV];
    load_chunk<T, NV>(z, (const T*)a.logits + (size_t)row * a.ld, lo, hi, ch.vec, s.inv);
    if (!s.k && s.P >= (1u << 30)) {  // no cut along the order: what min-p keeps
        uint64_t sum = 0;
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (j * CT * 4 < n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint64_t w = score_weight(z[j][e], m);
                    sum += w >= s.least ? 1ull << PACK | w : 0;
                }
        sum = block_reduce<CT>(l, sum, (uint64_t)0, Sum{});
        if (tid == 0) r.sure[blockIdx.x] = sum;
        return;
    }
    for (int i = tid; i < BINS; i += CT) t[i] = 0;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < NV; ++j)
        if (j * CT * 4 < n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const unsigned d = dist_bits(z[j][e], m);
                if (d < DMAX) atomicAdd(&t[bin_of(d)], 1ull << PACK | score_weight(z[j][e], m));
            }
    __syncthreads();
    for (int i = tid; i < BINS; i += CT) {
        r.bins(blockIdx.x)[i] = t[i];
        if (t[i]) {
            atomicAdd(&r.t.cnt[i], (unsigned)(t[i] >> PACK));
            atomicAdd(&r.t.mass[i], t[i] & LOW);
        }
    }
}

static __device__ __forceinline__ Plan plan_of(const Tally& t, const Setting& s) {  // by one wave
    Scan<BINS> scan;
    scan.make(t.mass, t.cnt, BINS, 0, 0);
    Plan p{BINS, BINS, -1, true, true};
    Found k{-1, 0, 0, 0, 0};
    if (s.k) k = scan.find(s.k, true);
    if (k.bin >= 0) p.lo = p.hi = p.k = k.bin;
    if (s.P < (1u << 30)) {  // no later than if all of top-k's last bin counted, and no earlier than if none of it did
        p.hi = scan.find(top_p_need(s.P, k.bin < 0 ? scan.mt : k.mass + k.in_mass), false).bin;
        p.lo = k.bin < 0 ? p.hi : scan.find(top_p_need(s.P, k.mass), false).bin;
    }
    p.order = p.lo < BINS;
    // Where min-p ends, or the weights themselves (least == 1): near the distance of that weight.  The weights' polynomial and roundings move it by less than
    // 1e-6 up to 1e-3 and by less than a bin behind that.  Near 2^32 by what the weight lacks: one unit of the logarithm of the weight itself would be 1.3e-6
    // there, ten of the bins.  (A logarithm in 64 bits: the launch 0.4 us longer.)
    const float d = s.least > 1ull << 31 ? -log1pf((float)((1ull << 32) - s.least) * -0x1p-32f) : (32.f - log2f((float)s.least)) * 0.693147181f;
    auto bin_near = [](float x) { return bin_of(min(__float_as_uint(fmaxf(x, 0.f)), DMAX - 1)); };
    const int b0 = max(bin_near(d - 2e-6f) - 1, 0), b1 = min(bin_near(d + 2e-6f) + 1, BINS - 1);
    if (b1 < p.lo) p = Plan{b0, b1, -1, false, true};  // before everything else ends: it alone counts
    else p.lo = min(p.lo, b0);                         // (behind hi: nothing changes)
    unsigned n = 0;
#pragma unroll
    for (int i = 0; i < Scan<BINS>::E; ++i) {
        const int b = (threadIdx.x & 63) * Scan<BINS>::E + i;
        n += b < BINS && ((b >= p.lo && b <= p.hi) || b == p.k) ? t.cnt[b] : 0;
    }
    p.fits = wave_all(n, 0u, Sum{}) <= LIST;
    return p;
}
template <int NT>
static __device__ __forceinline__ void fetch_tally(Tally& t, const RowState& r) {
    for (int i = threadIdx.x; i < BINS; i += NT) {
        t.mass[i] = r.t.mass[i];
        t.cnt[i] = r.t.cnt[i];
    }
}

template <typename T, int NV>
__global__ void __launch_bounds__(CT, 4) chunk_list_kernel(const CutArgs a, const ChunkArgs ch) {
    __shared__ struct {
        unsigned long long red[CT / 64];
        unsigned at;
    } l;
    __shared__ Tally t;
    __shared__ Plan plan;
    __shared__ Entry stage[STAGE];
    __shared__ unsigned n_stage;
    const int row = blockIdx.y, tid = threadIdx.x;
    const Setting s = setting_of(a.how, row);
    if (!s.k && s.P >= (1u << 30)) return;
    RowState& r = ch.row(row);
    bool settled;
    const float m = row_max(r, ch.chunks, by_chunks(s, ch), settled);
    if (settled || !s.ok || !(m > -INFINITY)) return;
    const int lo = blockIdx.x * ch.chunk, hi = min(a.vocab, lo + ch.chunk), n = hi - lo;
    fetch_tally<CT>(t, r);
    f32x4 z[NV];
    load_chunk<T, NV>(z, (const T*)a.logits + (size_t)row * a.ld, lo, hi, ch.vec, s.inv);
    __syncthreads();
    if (tid < 64) {  // (all four waves would take the compute unit's time from other workgroups)
        const Plan p = plan_of(t, s);
        if (tid == 0) {
            n_stage = 0;
            plan = p;
            if (blockIdx.x == 0) r.plan = p;
        }
    }
    __syncthreads();
    const Plan pl = plan;
    uint64_t sum = 0;  // of the chunk's own bins below lo
#pragma unroll
    for (int i = 0; i < (BINS + CT - 1) / CT; ++i) sum += i * CT + tid < pl.lo ? r.bins(blockIdx.x)[min(i * CT + tid, BINS - 1)] : 0;
    sum = block_reduce<CT>(l, sum, (uint64_t)0, Sum{});
    if (tid == 0) r.sure[blockIdx.x] = sum;
    if (!pl.fits) return;
#pragma unroll
    for (int j = 0; j < NV; ++j)
        if (j * CT * 4 < n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const unsigned d = dist_bits(z[j][e], m);
                if (d >= DMAX) continue;
                const int b = bin_of(d);
                if ((b >= pl.lo && b <= pl.hi) || b == pl.k) {
                    unsigned at = atomicAdd(&n_stage, 1u);
                    Entry* to = stage;
                    if (at >= STAGE) {
                        at = atomicAdd(&r.listed, 1u);
                        to = r.list;
                    }
                    to[at] = Entry{z[j][e], (unsigned)(lo + (j * CT + tid) * 4 + e)};
                }
            }
    __syncthreads();
    const unsigned mine = min(n_stage, (unsigned)STAGE);
    if (tid == 0 && mine) l.at = atomicAdd(&r.listed, mine);
    __syncthreads();
    for (unsigned i = tid; i < mine; i += CT) r.list[l.at + i] = stage[i];
}

constexpr int FT = 512, SUB = 4096, NB = (CHUNK_MOST + FT * 4 - 1) / (FT * 4);
struct Weighed {
    unsigned long long w;
    float z;
    unsigned idx;
};
template <typename T>
__global__ void __launch_bounds__(FT) row_end_kernel(const CutArgs a, const ChunkArgs ch) {
    __shared__ CutLds<FT> l;
    __shared__ Tally t;
    __shared__ union {
        Entry list[LIST];
        struct {
            float z[LIST];
            Weighed sub[SUB];
        };
    } u;
    __shared__ unsigned long long cm[CHUNKS], bw[NB * FT / 64];
    __shared__ unsigned own[CHUNKS], n_sub;
    const int row = blockIdx.x, tid = threadIdx.x, vocab = a.vocab, chunks = ch.chunks;
    const Setting s = setting_of(a.how, row);
    RowState& r = ch.row(row);
    const T* p = (const T*)a.logits + (size_t)row * a.ld;
    bool settled;
    const float m = row_max(r, chunks, by_chunks(s, ch), settled);
    RowCut c = uncut(s, m);
    if (!s.ok || !(m > -INFINITY)) {
        if (tid == 0) {
            if (a.cut) a.cut[row] = c;
            if (a.u) emit(a, row, -1, 0, 0, 0);
        }
        return;
    }
    auto clear = [&]() {
        for (int i = tid; i < BINS; i += FT) {
            t.mass[i] = 0;
            t.cnt[i] = 0;
        }
    };
    auto from_row = [&](auto&& fn) {
        for (int i0 = 0; i0 < vocab; i0 += FT * 4) {
            const int i = i0 + tid * 4;
            f32x4 x{NAN, NAN, NAN, NAN};
            if (ch.vec && i + 4 <= vocab) x = logits4(p + i);
            else
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (i + e < vocab) x[e] = logit(p, i + e);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (i + e < vocab) fn(mul_once(x[e], s.inv), (unsigned)(i + e));
        }
    };
    // ---- a row that its chunks settled: of their lists only what reaches the row's own k-th bin; weights once ----
    if (settled) {
        const int most = own_most(chunks);
        unsigned long_ = 0;
        for (int i = tid & 63; i < chunks; i += 64) long_ = max(long_, r.own[i]);
        for (int o = 32; o > 0; o >>= 1) long_ = max(long_, (unsigned)__shfl_xor((int)long_, o, FS_WAVE));
        const int each_of = uniform((int)long_), all = each_of * chunks;  // entry i of chunk c at c * each_of + i; what a shorter list lacks weighs nothing
        if (tid < chunks) own[tid] = r.own[tid];
        if (tid == 0) {
            n_sub = 0;
            l.fn = 0;
        }
        clear();
        __syncthreads();
        for (int i0 = 0; i0 < all; i0 += FT * 8) {
            float z[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int i = i0 + k * FT + tid, c = min(i / each_of, chunks - 1), e = i - c * each_of;
                z[k] = i < all && e < (int)own[c] ? r.list[c * most + e].z : NAN;
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int i = i0 + k * FT + tid;
                if (i < all) u.z[i] = z[k];
                const unsigned d = dist_bits(z[k], m);
                if (d < DMAX) atomicAdd(&t.cnt[bin_of(d)], 1u);
            }
        }
        __syncthreads();
        Scan<BINS> scan;
        scan.make(t.mass, t.cnt, BINS, 0, 0);
        const Found f = scan.find(s.k, true);
        const int last = f.bin < 0 ? BINS : f.bin;
        const unsigned few = f.cnt + f.in_cnt;
        if (few <= SUB) {
            for (int i = tid; i < all; i += FT) {
                const unsigned d = dist_bits(u.z[i], m);
                if (d < DMAX && bin_of(d) <= last) u.sub[atomicAdd(&n_sub, 1u)].idx = i;
            }
            __syncthreads();
            const int n = uniform((int)n_sub);
            for (int j = tid; j < n; j += FT) {
                const int i = (int)u.sub[j].idx, c = i / each_of;
                const float z = u.z[i];
                const unsigned idx = r.list[c * most + i - c * each_of].idx;
                if (n <= FEW) {
                    l.fz[j] = z;
                    l.fi[j] = idx;
                } else {
                    const uint64_t w = score_weight(z, m);
                    u.sub[j] = Weighed{w, z, idx};
                    atomicAdd(&t.mass[bin_of(dist_bits(z, m))], (unsigned long long)w);
                }
            }
            if (tid == 0) l.fn = n;
            __syncthreads();
            if (n <= FEW) {
                few_end<FT>(l, a, row, s, c);
                return;
            }
            auto each = [&](auto&& fn) {
                for (int i = tid; i < n; i += FT) fn(u.sub[i].z, u.sub[i].idx);
            };
            cut_along<FT>(l, t, a, row, s, false, each, c);
            uint64_t R = 0;
            unsigned kept = 0;
            for (int i = tid; i < n; i += FT) {
                Weighed& e = u.sub[i];
                if (!(e.w >= s.least && (e.z > c.z || (e.z == c.z && e.idx <= c.idx)))) e.w = 0;
                R += e.w;
                kept += e.w != 0;
            }
            R = block_reduce<FT>(l, R, (uint64_t)0, Sum{});
            kept = block_reduce<FT>(l, kept, 0u, Sum{});
            c.R = R;
            if (a.cut && tid == 0) a.cut[row] = c;
            if (!a.u) return;
            const Bound b = select_index<FT>(l, draw_target(a, row, R), kept, [&](auto&& fn) {
                for (int i = tid; i < n; i += FT)
                    if (u.sub[i].w) fn(u.sub[i].w, u.sub[i].idx);
            });
            if (tid == 0) emit(a, row, (int)b.idx, b.mass, R, kept);
            return;
        }
    }
    // ---- others: the listed bins beside the chunks' sums, or, where a list does not hold them (rows with thousands of nearly equal scores) or nothing was
    // listed, the row in memory ----
    const bool along = s.k || s.P < (1u << 30), sums = !settled && ch.later;
    Plan pl{along ? 0 : BINS, BINS, -1, along, false};
    int n = 0;
    if (sums && along) {
        fetch_tally<FT>(t, r);
        pl = r.plan;
        n = pl.fits ? (int)r.listed : 0;
        for (int i = tid; i < n; i += FT) u.list[i] = r.list[i];
    } else if (along) {
        __syncthreads();
        clear();
        __syncthreads();
        from_row([&](float z, unsigned) { count_in(t, z, m); });
    }
    unsigned kept = 0;
    if (tid < CHUNKS) {
        const unsigned long long x = sums && tid < chunks ? r.sure[tid] : 0;
        cm[tid] = x & LOW;
        kept = (unsigned)(x >> PACK);
    }
    auto each = [&](auto&& fn) {
        if (pl.fits)
            for (int i = tid; i < n; i += FT) fn(u.list[i].z, u.list[i].idx);
        else
            from_row(fn);
    };
    __syncthreads();
    if (pl.order) cut_along<FT>(l, t, a, row, s, false, each, c);
    if (pl.lo < BINS)
        each([&](float z, unsigned i) {
            const uint64_t w = cut_weight(c, z, i);
            if (!w || bin_of(dist_bits(z, m)) < pl.lo) return;
            atomicAdd(&cm[i / ch.chunk], (unsigned long long)w);
            ++kept;
        });
    kept = block_reduce<FT>(l, kept, 0u, Sum{});
    // (every wave by itself; what the kept scores of the list add to the chunks stands behind the barriers of the sum above)
    const int lane = tid & 63, wv = uniform(tid >> 6);
    constexpr int CE = CHUNKS / 64;
    uint64_t own_m = 0, cmass[CE];
#pragma unroll
    for (int i = 0; i < CE; ++i) own_m += cmass[i] = cm[lane * CE + i];
    const uint64_t upto_m = wave_upto(own_m, (uint64_t)0, Sum{}), R = of_lane(upto_m, 63);
    c.R = R;
    if (a.cut && tid == 0) a.cut[row] = c;
    if (!a.u) return;
    const uint64_t target = draw_target(a, row, R);
    const int from = __ffsll(__ballot(upto_m > target)) - 1;
    uint64_t base = of_lane(upto_m - own_m, from);
    int at = from * CE;
#pragma unroll
    for (int i = 0; i < CE - 1; ++i)
        if (at == from * CE + i) {
            const uint64_t x = of_lane(cmass[i], from);
            if (base + x <= target) {
                base += x;
                ++at;
            }
        }
    // the chunk in blocks of four scores per thread: a sum for each wave's part of each block, then the wave that holds the target looks on
    const int c0 = at * ch.chunk, c1 = min(vocab, c0 + ch.chunk);
    f32x4 x[NB];
    uint64_t run[NB] = {};
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        const int i = c0 + (j * FT + tid) * 4;
        x[j] = f32x4{NAN, NAN, NAN, NAN};
        if (ch.vec && i + 4 <= c1) x[j] = logits4(p + i);
        else
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (i + e < c1) x[j][e] = logit(p, i + e);
    }
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        if (c0 + j * FT * 4 >= c1) {
            if (lane == 63) bw[j * (FT / 64) + wv] = 0;
            continue;
        }
        uint64_t sum = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) sum += cut_weight(c, mul_once(x[j][e], s.inv), c0 + (j * FT + tid) * 4 + e);
        run[j] = wave_upto(sum, (uint64_t)0, Sum{});
        if (lane == 63) bw[j * (FT / 64) + wv] = run[j];
    }
    __syncthreads();
    static_assert(NB * FT / 64 <= 64, "one part of a block to a lane");
    const uint64_t part = lane < NB * FT / 64 ? bw[lane] : 0, upto = wave_upto(part, (uint64_t)0, Sum{});
    const int k = __ffsll(__ballot(base + upto > target)) - 1;
    base += of_lane(upto - part, k);
    if (wv != k % (FT / 64)) return;
#pragma unroll
    for (int j = 0; j < NB; ++j)
        if (j == k / (FT / 64)) {
            uint64_t w[4], sum = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                w[e] = cut_weight(c, mul_once(x[j][e], s.inv), c0 + (j * FT + tid) * 4 + e);
                sum += w[e];
            }
            uint64_t before = base + run[j] - sum;
            if (before <= target && target < before + sum) {
                int e = 0;
                while ((before += w[e]) <= target) ++e;
                emit(a, row, c0 + (j * FT + tid) * 4 + e, w[e], R, kept);
            }
        }
}

constexpr int ROW_MOST = 8192;  // longest row that one workgroup takes alone

// Short chunks, many workgroups: rows differ in what they need, and a workgroup's fixed work is small.  Us a call in chunks of up to 4096 and of up to 12288: one
// row x 152064 top-k 50 13.1, 15.6, top-p 30.2, 40.1; 64 rows top-p 59.2, 63.1, top-k 300 58.6, 40.0 (12288: its lists still hold it); 300 rows top-p
// 163, 171.  Beyond some thousands of workgroups longer ones, for the scratch (390 KB a row of 152064 in the short ones, 230 in the long).
constexpr int FINE_WGS = 16384;
int fine_chunks(int vocab) { return (vocab + CHUNK_LEAST - 1) / CHUNK_LEAST; }
int row_chunks(int rows, int vocab) {
    const int fine = fine_chunks(vocab);
    return (long long)rows * fine <= FINE_WGS ? fine : (vocab + CHUNK_MOST - 1) / CHUNK_MOST;
}

template <typename T, int NV>
void launch_chunks(const CutArgs& a, const ChunkArgs& ch, int k, hipStream_t s) {
    const CutSettings& h = a.how;
    const dim3 g(ch.chunks, a.rows);
    hipLaunchKernelGGL((chunk_top_kernel<T, NV>), g, dim3(CT), 0, s, a, ch);
    if (!ch.later) return;
    hipLaunchKernelGGL((chunk_bins_kernel<T, NV>), g, dim3(CT), 0, s, a, ch);
    const bool order = h.temperature || h.top_k || h.top_p || k > 0 || h.top_p_all < 1.f;
    if (order) hipLaunchKernelGGL((chunk_list_kernel<T, NV>), g, dim3(CT), 0, s, a, ch);
}

template <typename T>
hipError_t launch(const CutArgs& a, void* work, hipStream_t s) {
    const bool vec = a.ld % 4 == 0 && a.vocab % 4 == 0 && ((uintptr_t)a.logits & (4 * sizeof(T) - 1)) == 0;
    if (a.vocab <= ROW_MOST) {
        const dim3 g(a.rows);
        if (a.vocab <= 2048) hipLaunchKernelGGL((cut_row_kernel<T, 256, 2048>), g, dim3(256), 0, s, a, vec);
        else hipLaunchKernelGGL((cut_row_kernel<T, 512, ROW_MOST>), g, dim3(512), 0, s, a, vec);
        return hipGetLastError();
    }
    ChunkArgs ch{(char*)work, 0, 0, row_chunks(a.rows, a.vocab), vec, true};
    ch.chunk = ((a.vocab + ch.chunks - 1) / ch.chunks + 3) & ~3;
    ch.chunks = (a.vocab + ch.chunk - 1) / ch.chunk;
    ch.stride = row_bytes(ch.chunks);
    // one top-k for all rows that their chunks can settle: nothing else follows
    const CutSettings& h = a.how;
    const int k = !h.temperature && h.temperature_all == 0.f ? 1 : h.top_k ? 0 : h.top_k_all;
    ch.later = k < 1 || k > top_most(ch.chunks);
    if (ch.chunk <= CHUNK_LEAST) launch_chunks<T, 4>(a, ch, k, s);
    else launch_chunks<T, 12>(a, ch, k, s);
    hipLaunchKernelGGL(row_end_kernel<T>, dim3(a.rows), dim3(FT), 0, s, a, ch);
    return hipGetLastError();
}

}  // namespace

// (scratch for many rows serves few ones too, which are in short chunks: the most rows of those can need more than the rows given)
size_t cut_workspace_bytes(int rows, int vocab) {
    if (vocab <= ROW_MOST) return 256;
    const int fine = std::min(rows, FINE_WGS / fine_chunks(vocab));
    return std::max((size_t)rows * row_bytes(row_chunks(rows, vocab)), (size_t)fine * row_bytes(fine_chunks(vocab)));
}

hipError_t launch_cut(int dtype, const CutArgs& a, void* work, hipStream_t s) { return dtype == 0 ? launch<float>(a, work, s) : launch<bf16_t>(a, work, s); }
