// Attention of draft-tree segments against a context whose settled tokens lie in pages of 64, 8 bits each (e4m3, a power-of-two scale
// per page, K or V, head), and whose newest slots lie in the 16- or 32-bit cache.
//
// The rows of the G query heads that share a KV head are stacked (R = G * M), as in the tree-attention kernel.  Grid: (split, KV head,
// request x row block); a workgroup has one group of four waves, or two, with 16 or 32 rows each; a group's waves take alternate pages, so nothing
// is shared until the end and no wave waits for another.  A page is stored in matrix-operand order: every lane loads its 16 codes of
// a fragment pair straight into registers (1 KiB per wave and load) and one instruction turns two codes into two bf16 values, times
// the scale, exactly (4 significant bits, a power of two).  What is multiplied is what the page stands for; nothing is rounded.
// The waves' sums meet in LDS, those of the splits in paged_merge_kernel, both in a fixed order.
//
// Bound: the stream of the pages, 1 byte per element, half of what a 16-bit cache takes (64 rows behind 16k slots, 32 heads of 128: 137 MB in
// 34.5 us, 4.0 TB/s, 1.02 of the algorithmic bytes; short contexts: latency, 8.8 us for one row behind 1000 slots; medians of 60 traced launches).  Every
// block of 64 rows reads and expands the pages anew, so a segment of many blocks is the slower over pages (1024 rows behind 4096 slots, 32 heads of 128:
// 171 us a layer, the tree attention over the 16-bit cache 131; 64 rows behind 16k slots 39 and 57).
#include "paged.hpp"
#include "rows_attn.hpp"

#include <algorithm>
#include <type_traits>

namespace {

constexpr int STREAMS = 4;  // waves of the same rows, which take every fourth page

template <typename T>
struct Codes;
template <>
struct Codes<bf16_t> {
    typedef __bf16 pair_t __attribute__((ext_vector_type(2)));
    // 8 codes (two words) times 2^e -> one fragment
    static __device__ __forceinline__ bf16x8 frag(const unsigned* w, float scale) {
        bf16x8 f;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const pair_t lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, false);
            const pair_t hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, true);
            f[4 * i] = lo[0];
            f[4 * i + 1] = lo[1];
            f[4 * i + 2] = hi[0];
            f[4 * i + 3] = hi[1];
        }
        return f;
    }
};
template <>
struct Codes<float> {
    typedef float pair_t __attribute__((ext_vector_type(2)));
    static __device__ __forceinline__ f32x4 frag(const unsigned* w, float scale) {  // 4 codes
        const pair_t lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[0], scale, false);
        const pair_t hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[0], scale, true);
        return f32x4{lo[0], lo[1], hi[0], hi[1]};
    }
};

// Whether a stacked row sees no slot at all (a zero row then; otherwise a zero sum is 0 / 0 as the formula has it).
static __device__ __forceinline__ bool sees_nothing(const PagedBase& a, const PagedReq& rq, int row) {
    if (rq.l_glo > 0 || !a.anc) return false;
    const int T = rq.seg_off + rq.M;
    const uint64_t* w = a.anc + (size_t)row * FS_ANC_WORDS;
    for (int i = 0; i * 64 < T; ++i) {
        const int left = T - i * 64;
        if (w[i] & (left >= 64 ? ~0ull : (1ull << left) - 1)) return false;
    }
    return true;
}

// Work over a request's context: its pages, and `tw` for every 64 slots behind them.
static __host__ __device__ __forceinline__ int units_of(const PagedReq& r, int tw) {
    return (r.n_paged + PAGE_TOK - 1) / PAGE_TOK + (r.l_glo + r.seg_off + r.M - r.n_paged + 63) / 64 * tw;
}

template <typename T>
static __device__ __forceinline__ void store_row(const PagedBase& a, const PagedReq& rq, int kvh, int loc, int c, const f32x4& o, float den) {
    using E = Elem<T>;
    const int row = rq.row0 + loc % rq.M, qh = kvh * a.G + loc / rq.M;
    float inv = 1.0f / den;
    f32x4 v = o * inv;
    if (den == 0.f && sees_nothing(a, rq, row)) v = f32x4{0.f, 0.f, 0.f, 0.f};
    T* p = a.ldo ? (T*)a.o + (size_t)row * a.ldo + (size_t)qh * a.hd + c
                 : (T*)a.o + frag_major_index<T>(row, qh * a.hd + c, a.Hq * a.hd / E::KT);
    *(typename E::out4_t*)p = E::pack4(v[0], v[1], v[2], v[3]);
}

// What a tile of 64 slots behind the pages costs, in pages: a round of the waves is four pages, or two halves of one such tile for every row tile.
static __host__ __device__ constexpr int tail_weight(int mtw) { return mtw == 1 ? 2 : 4; }

// RG groups of MTW row tiles each; every page is read by the RG waves that share it, one after the other from the caches.  (16 bits: the bound
// of 512 threads also where there are 256 keeps a wave's registers in one file, two waves to a SIMD.)
// SHARED: a pass over part of the contexts, from a page on and up to a slot, whose sums are partial always.
template <typename T, int HD, int MTW, int RG, bool APART, bool SHARED>
__global__ void __launch_bounds__(sizeof(T) == 2 ? 512 : 256) paged_attn_kernel(const std::conditional_t<SHARED, SharedArgs, PagedArgs> a) {
    constexpr int PW = STREAMS * RG, TW = APART ? STREAMS : PW;  // waves over pages, waves over the slots behind them
    constexpr int WAVES = APART ? PW + TW : PW;
    static_assert(!APART || RG == 1, "waves of one group");
    using RT = RowTiles<T, HD, MTW>;
    using frag_t = typename RT::frag_t;
    constexpr int NA = HD / 64, NHT = HD / 16, PER = RT::PER;
    constexpr int RROW = HD + 4;  // padded row of the sums that the waves exchange
    constexpr int WPR = STREAMS / MTW;  // waves that share a row tile behind the pages
    using TT = RowTiles<T, HD, 1>;
    constexpr int LDS_STAGE = TW * TT::STAGE * (int)sizeof(T), LDS_RED = PW * 16 * (RROW + 2) * 4;
    __shared__ __align__(16) unsigned char lds[LDS_STAGE > LDS_RED ? LDS_STAGE : LDS_RED];
    constexpr int NKT = RT::NKT, QT = MTW * RG * NKT;  // fragments of the workgroup's queries
    __shared__ __align__(16) unsigned char q_lds[QT * 1024];
    __shared__ __align__(16) float tail_o[TW * 16 * (RROW + 2)];  // the sums over the slots behind the pages: [wave][row][RROW], then (m, l)

    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r16 = lane & 15, g = lane >> 4;
    const int split = blockIdx.x, kvh = blockIdx.y, rqi = blockIdx.z / a.row_blocks, rb = blockIdx.z % a.row_blocks;
    const auto rq = a.req[rqi];
    const int M = rq.M, R = a.G * M, rho0 = rb * 16 * MTW * RG;
    if (rho0 >= R) return;  // a shorter request of the batch has no such row block
    int L, first_page = 0;  // (pages are counted from first_page on below)
    if constexpr (SHARED) {
        L = rq.L;
        first_page = rq.first;
    } else {
        L = rq.l_glo + rq.seg_off + M;
    }
    const int np = (rq.n_paged + PAGE_TOK - 1) / PAGE_TOK - first_page, nt = (L - rq.n_paged + 63) / 64;
    // the split's share: pages are one unit each, tiles of 64 slots behind them tail_weight(MTW)
    const int u0 = split * a.units_per_split, u1 = u0 + a.units_per_split, tw = tail_weight(MTW);
    if (u0 >= np + nt * tw) return;  // a shorter context has no such split
    const int t0 = min(u0, np), tp = min(u1, np);
    const int j0 = u0 <= np ? 0 : (u0 - np + tw - 1) / tw, j1 = u1 <= np ? 0 : min(nt, (u1 - np + tw - 1) / tw);
    // the queries as fragments, one KiB each
    for (int f = w; f < QT; f += WAVES) {
        const int rho = rho0 + f / NKT * 16 + r16, rr = rho < R ? rho : 0;
        const T* qp = (const T*)a.q + (size_t)(rq.row0 + rr % M) * a.ldq + (size_t)(kvh * a.G + rr / M) * HD;
        *(frag_t*)(q_lds + f * 1024 + lane * 16) = rho < R ? *(const frag_t*)(qp + RT::col(f % NKT, g)) : RT::E::zero();
    }
    __syncthreads();
    // ---- slots behind the pages, in the cache: halves of 32, masked where they hold draft slots.  A wave takes one row tile and every
    // WPR-th half; its sums wait in LDS for the others', so that they take no registers from the part below ----
    const bool tail = j1 > j0;
    const int tw_id = APART ? w - PW : w;  // (apart: waves of their own do this while the others are at the pages)
    if (tail && tw_id >= 0) {
        const int w = tw_id;
        TT rt;
        rt.init();
        const int rho = rho0 + w % (MTW * RG) * 16 + r16, seg_r = rho % M;
        const bool rok = rho < R;
#pragma unroll
        for (int kt = 0; kt < NKT; ++kt) rt.qf[0][kt] = *(const frag_t*)(q_lds + (w % (MTW * RG) * NKT + kt) * 1024 + lane * 16);
        const T* kbase = (const T*)rq.tail + a.layer_off + (size_t)kvh * a.stride_head;
        T* vt = (T*)lds + w * TT::STAGE;
        for (int x = 2 * j0 + w / (MTW * RG); x < 2 * j1; x += WPR) {
            const int s0 = rq.n_paged + x * 32;
            if (s0 >= L) break;
            const int valid = min(L - s0, 32), d0 = s0 - rq.l_glo;
            const unsigned in = valid == 32 ? ~0u : (1u << valid) - 1;
            unsigned m = ~0u;
            if (d0 + 32 > 0) {  // some of the slots are draft slots: slot s0 + b is S index d0 + b
                if (a.anc) {
                    const uint64_t* am = a.anc + (size_t)(rq.row0 + seg_r) * FS_ANC_WORDS;
                    if (d0 >= 0) {
                        const int wd = d0 >> 6, sh = d0 & 63;
                        uint64_t y = am[wd] >> sh;
                        if (sh > 32 && wd + 1 < FS_ANC_WORDS) y |= am[wd + 1] << (64 - sh);
                        m = (unsigned)y;
                    } else {
                        m = (unsigned)(((1ull << -d0) - 1) | (am[0] << -d0));
                    }
                } else {
                    const int n = rq.seg_off + seg_r + 1 - d0;  // a chain: S indices up to the row's own
                    m = n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1;
                }
            }
            const unsigned vis[1] = {rok ? m & in : 0u};
            if (__ballot(vis[0] != 0) == 0) continue;
            const T* kp = kbase + (long long)(s0 - rq.n_paged) * a.stride_tok;
            if (__ballot(rok && vis[0] != ~0u) != 0)
                rt.template half<true>(kp, kp + a.stride_kv, a.stride_tok, a.stride_tok, valid - 1, vis, a.scale_log2, vt, lane);
            else
                rt.template half<false>(kp, kp + a.stride_kv, a.stride_tok, a.stride_tok, valid - 1, vis, a.scale_log2, vt, lane);
        }
        const float l = rt.row_sum(0);
#pragma unroll
        for (int n = 0; n < NHT; ++n) *(f32x4*)(tail_o + (w * 16 + r16) * RROW + n * 16 + g * 4) = rt.acc[0][n];
        if (g == 0) *(float2*)(tail_o + TW * 16 * RROW + (w * 16 + r16) * 2) = make_float2(rt.m[0], l);
    }

    // ---- settled pages: the wave's tiles t0 + ps, + 4, ...; the next one's K and V codes are on their way while one is computed ----
    RT rt;
    rt.init();
    bool bad = false;
    const int rg = w % RG, ps = w / RG;
    if (w < PW && t0 + ps < tp) {
        // ids and scales by scalar loads: they do not stand in the way of the waits for codes (nothing writes them while the kernel runs)
        typedef const __attribute__((address_space(4))) int32_t* cint_p;
        typedef const __attribute__((address_space(4))) float* cfloat_p;
        const cint_p ids = (cint_p)(a.table + (size_t)rq.seq * a.max_pages + first_page);
        const cfloat_p scales = (cfloat_p)a.scales;
        const int lane16 = r16 * 4 + g;  // the lane's 16 bytes of a KiB in operand order
        const unsigned char* ql = q_lds + rg * MTW * NKT * 1024 + lane * 16;
        u32x4 kc[4][NA], vc[NHT];
        float ks, vs;
        // an id outside the pool: page 0 is read in its place and the rows become NaN
        auto page_id = [&](int raw) {
            const int id = __builtin_amdgcn_readfirstlane(raw);  // (uniform)
            const bool ok = (unsigned)id < (unsigned)a.n_pages;
            bad |= !ok;
            return ok ? id : 0;
        };
        auto k_tile = [&](int id) { return (long long)id * a.page_tiles + a.tile0 + kvh; };
        auto load_k = [&](long long tile) __attribute__((always_inline)) {
            const u32x4* p = (const u32x4*)(a.codes + tile * (PAGE_TOK * HD)) + lane16;
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int c = 0; c < NA; ++c) kc[j][c] = *(p + c * 256 + j * 64);
            ks = scales[tile];
        };
        auto load_v = [&](long long tile) __attribute__((always_inline)) {
            const u32x4* p = (const u32x4*)(a.codes + tile * (PAGE_TOK * HD)) + lane16;
#pragma unroll
            for (int n = 0; n < NHT; ++n) vc[n] = *(p + n * 64);
            vs = scales[tile];
        };
        f32x4 st[MTW][4];
        auto scores = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < MTW; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) st[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < NA; ++c)
#pragma unroll
                for (int h = 0; h < PER; ++h) {
                    frag_t qv[MTW];
#pragma unroll
                    for (int i = 0; i < MTW; ++i) qv[i] = *(const frag_t*)(ql + (i * NKT + c * PER + h) * 1024);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const unsigned wd[4] = {kc[j][c][0], kc[j][c][1], kc[j][c][2], kc[j][c][3]};
                        const frag_t kf = Codes<T>::frag(wd + h * (4 / PER), ks);
#pragma unroll
                        for (int i = 0; i < MTW; ++i) st[i][j] = RT::E::mma(kf, qv[i], st[i][j]);
                    }
                    __builtin_amdgcn_sched_barrier(0);  // (keeps the codes from being expanded all at once)
                }
        };
        auto products = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int jj = 0; jj < 4 / RT::NSUB; ++jj) {
                frag_t pf[MTW];
#pragma unroll
                for (int i = 0; i < MTW; ++i) pf[i] = RT::template pack_p<4>(st[i], jj);
#pragma unroll
                for (int n = 0; n < NHT; ++n) {
                    const unsigned wd[2] = {vc[n][jj * RT::NSUB], vc[n][(jj * RT::NSUB + RT::NSUB - 1)]};
                    const frag_t vf = Codes<T>::frag(wd, vs);
#pragma unroll
                    for (int i = 0; i < MTW; ++i) rt.acc[i][n] = RT::E::mma(vf, pf[i], rt.acc[i][n]);
                    if (n & 1) __builtin_amdgcn_sched_barrier(0);
                }
            }
        };
        const int whole = min(tp, rq.n_paged / PAGE_TOK - first_page);  // (only the last page of a context can be partial)
        int t = t0 + ps;
        const long long first = k_tile(page_id(ids[t]));
        int ahead = ids[t + STREAMS < tp ? t + STREAMS : t];  // (in the loop's order, so that its waits can count)
        load_k(first);
        load_v(first + a.Hkv);
        for (; t < whole; t += STREAMS) {
            // behind the wave's last tile the same one is fetched once more, from the caches: no load hangs on a branch
            const long long next = k_tile(page_id(ahead));
            ahead = ids[t + 2 * STREAMS < tp ? t + 2 * STREAMS : t];
            scores();
            load_k(next);
#pragma unroll
            for (int i = 0; i < MTW; ++i) rt.template softmax<4, false>(i, st[i], a.scale_log2, 0ull);
            products();
            load_v(next + a.Hkv);
        }
        if (t < tp) {  // the partial page
            const int cnt = rq.n_paged - (first_page + t) * PAGE_TOK;
            const unsigned long long vis = ((1ull << cnt) - 1) >> (g * 4);
            scores();
#pragma unroll
            for (int i = 0; i < MTW; ++i) rt.template softmax<4, true>(i, st[i], a.scale_log2, vis);
            // tokens behind the settled ones count for nothing, whatever their codes
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int n = min(max(cnt - (q * 16 + g * 4), 0), 4);
                const unsigned keep = n == 4 ? ~0u : (1u << (8 * n)) - 1;
#pragma unroll
                for (int k = 0; k < NHT; ++k) vc[k][q] &= keep;
            }
            products();
        }
    }

    // ---- the waves' sums: one row tile of each group at a time through LDS ----
    float* ro = (float*)lds;              // [wave][row][RROW]
    float* rml = ro + PW * 16 * RROW;     // [wave][row][2]
    const float* tml = tail_o + TW * 16 * RROW;
#pragma unroll
    for (int i = 0; i < MTW; ++i) {
        if (rho0 + i * 16 >= R) break;  // uniform (the first group's rows come first)
        __syncthreads();
        if (w < PW) {
            const float l = bad ? __builtin_nanf("") : rt.row_sum(i);
#pragma unroll
            for (int n = 0; n < NHT; ++n) *(f32x4*)(ro + (w * 16 + r16) * RROW + n * 16 + g * 4) = rt.acc[i][n];
            if (g == 0) *(float2*)(rml + (w * 16 + r16) * 2) = make_float2(rt.m[i], l);
        }
        __syncthreads();
        const int row = tid >> 4 & 15, grp = tid >> 8, ti = grp * MTW + i, rho = rho0 + ti * 16 + row;
        if (grp >= RG || rho >= R) continue;
        // (the sums of the group's four waves over the pages, then of those that had this row tile behind them)
        float2 ml[STREAMS + WPR];
        float mm = FS_NEG_INF;
#pragma unroll
        for (int k = 0; k < STREAMS + WPR; ++k) {
            if (k < STREAMS) ml[k] = *(const float2*)(rml + ((k * RG + grp) * 16 + row) * 2);
            else ml[k] = tail ? *(const float2*)(tml + ((ti + MTW * RG * (k - STREAMS)) * 16 + row) * 2) : make_float2(FS_NEG_INF, 0.f);
            mm = fmaxf(mm, ml[k].x);
        }
        const float msub = mm == FS_NEG_INF ? 0.f : mm;
        float den = 0.f, wt[STREAMS + WPR];
#pragma unroll
        for (int k = 0; k < STREAMS + WPR; ++k) {
            wt[k] = __builtin_amdgcn_exp2f(ml[k].x - msub);
            den += wt[k] * ml[k].y;
        }
#pragma unroll
        for (int u = 0; u < NA; ++u) {
            const int c = (tid & 15) * 4 + u * 64;
            f32x4 o{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < STREAMS; ++k) o += *(const f32x4*)(ro + ((k * RG + grp) * 16 + row) * RROW + c) * wt[k];
            if (tail)
#pragma unroll
                for (int k = 0; k < WPR; ++k) o += *(const f32x4*)(tail_o + ((ti + MTW * RG * k) * 16 + row) * RROW + c) * wt[STREAMS + k];
            if (!SHARED && a.n_splits == 1) {
                store_row<T>(a, rq, kvh, rho, c, o, den);
            } else {
                size_t prow;
                if constexpr (SHARED) prow = ((size_t)(rq.part0 + split) * a.Hkv + kvh) * a.Rpad + (size_t)(rho / M) * a.rows + rq.row0 + rho % M;
                else prow = ((size_t)split * a.Hkv + kvh) * a.Rpad + (size_t)a.G * rq.row0 + rho;
                *(f32x4*)(a.part_o + prow * HD + c) = o;
                if (c == 0) *(float2*)(a.part_ml + prow * 2) = make_float2(mm, den);
            }
        }
    }
}

static __device__ __forceinline__ void merge_in(float& m, float& den, f32x4& o, const float2 ml, const f32x4 v) {
    const float mn = fmaxf(m, ml.x), ms = mn == FS_NEG_INF ? 0.f : mn;
    const float w0 = __builtin_amdgcn_exp2f(m - ms), w1 = __builtin_amdgcn_exp2f(ml.x - ms);
    den = den * w0 + ml.y * w1;
    o = o * w0 + v * w1;
    m = mn;
}
template <int LANES>
static __device__ __forceinline__ void merge_lanes(float& m, float& den, f32x4& o) {
#pragma unroll
    for (int x = 1; x < LANES; x <<= 1) {  // lane 0 of a group, whose sum is stored, always adds the higher lane's term second
        const float m2 = __shfl_xor(m, x, FS_WAVE), den2 = __shfl_xor(den, x, FS_WAVE);
        f32x4 o2;
#pragma unroll
        for (int e = 0; e < 4; ++e) o2[e] = __shfl_xor(o[e], x, FS_WAVE);
        merge_in(m, den, o, make_float2(m2, den2), o2);
    }
}

// out = sum_s 2^(m_s - m) O_s / sum_s 2^(m_s - m) l_s.  LANES adjacent lanes share four columns of a row and take splits q, q + LANES, ...,
// then meet pairwise in a fixed order.
template <typename T, int LANES>
__global__ void __launch_bounds__(256) paged_merge_kernel(const PagedArgs a) {
    const PagedReq rq = a.req[blockIdx.z];
    const int chunks = a.hd / 4, id = (blockIdx.x * 256 + threadIdx.x) / LANES, q = threadIdx.x % LANES;
    const int kvh = blockIdx.y, loc = id / chunks, c = id % chunks * 4, rho = a.G * rq.row0 + loc;
    if (loc >= a.G * rq.M) return;
    const int splits = (units_of(rq, a.tail_w) + a.units_per_split - 1) / a.units_per_split;
    const size_t step = (size_t)a.Hkv * a.Rpad, row = (size_t)kvh * a.Rpad + rho;
    float m = FS_NEG_INF, den = 0.f;
    f32x4 o{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = q; s < splits; s += LANES) {
        const float2 ml = *(const float2*)(a.part_ml + (row + s * step) * 2);
        const f32x4 v = *(const f32x4*)(a.part_o + (row + s * step) * a.hd + c);
        merge_in(m, den, o, ml, v);
    }
    merge_lanes<LANES>(m, den, o);
    if (q != 0) return;
    store_row<T>(a, rq, kvh, loc, c, o, den);
}

struct MergeGroups {
    int part0[PAGED_MAX_REQ], splits[PAGED_MAX_REQ];
};
// The same over a row's places: those of its group, then its own.
template <typename T, int LANES>
__global__ void __launch_bounds__(256) shared_merge_kernel(const SharedArgs a, const MergeGroups grp) {
    const SharedReq rq = a.req[blockIdx.z];
    const int chunks = a.hd / 4, id = (blockIdx.x * 256 + threadIdx.x) / LANES, q = threadIdx.x % LANES;
    const int kvh = blockIdx.y, loc = id / chunks, c = id % chunks * 4;
    if (loc >= a.G * rq.M) return;
    const int g0 = rq.group < 0 ? 0 : grp.part0[rq.group], gn = rq.group < 0 ? 0 : grp.splits[rq.group], all = gn + rq.splits;
    const size_t step = (size_t)a.Hkv * a.Rpad, row = (size_t)kvh * a.Rpad + (size_t)(loc / rq.M) * a.rows + rq.row0 + loc % rq.M;
    float m = FS_NEG_INF, den = 0.f;
    f32x4 o{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = q; s < all; s += LANES) {
        const size_t at = row + (size_t)(s < gn ? g0 + s : rq.part0 + s - gn) * step;
        merge_in(m, den, o, *(const float2*)(a.part_ml + at * 2), *(const f32x4*)(a.part_o + at * a.hd + c));
    }
    merge_lanes<LANES>(m, den, o);
    if (q != 0) return;
    store_row<T>(a, rq, kvh, loc, c, o, den);
}

// Workgroups a launch aims at, one per compute unit: each fetches alone what a unit can take in (16k slots, 64 rows, 32 heads: 8 splits 42 us, 16
// splits 51; 4k slots, 24 rows: 17.8 and 19.9).
constexpr int TARGET_WGS = 256;

template <typename T, int HD>
hipError_t launch(const PagedArgs& a, int row_tiles, hipStream_t s) {
    const dim3 grid(a.n_splits, a.Hkv, a.n_req * a.row_blocks);
    if constexpr (sizeof(T) == 2) {
        // Slots behind the pages by waves of their own where the launch leaves every workgroup a compute unit: they take as long as several pages
        // do, one after the other (one token behind 1000 slots: 10.0 -> 9.7 us; 32 tokens, 4 KV heads 20.3 -> 19.4); beyond that the waves would cost the
        // second workgroup of a unit (32 requests of 16 rows, 32 heads, 1k slots: 58.7 -> 63.0).
        const bool apart = (long long)grid.x * grid.y * grid.z <= TARGET_WGS;
        if (row_tiles == 1 && apart) hipLaunchKernelGGL((paged_attn_kernel<T, HD, 1, 1, true, false>), grid, dim3(512), 0, s, a);
        else if (row_tiles == 1) hipLaunchKernelGGL((paged_attn_kernel<T, HD, 1, 1, false, false>), grid, dim3(256), 0, s, a);
        else if (row_tiles == 2 && apart) hipLaunchKernelGGL((paged_attn_kernel<T, HD, 2, 1, true, false>), grid, dim3(512), 0, s, a);
        else if (row_tiles == 2) hipLaunchKernelGGL((paged_attn_kernel<T, HD, 2, 1, false, false>), grid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL((paged_attn_kernel<T, HD, 2, 2, false, false>), grid, dim3(512), 0, s, a);
    } else {
        hipLaunchKernelGGL((paged_attn_kernel<T, HD, 1, 1, false, false>), grid, dim3(256), 0, s, a);
    }
    if (a.n_splits > 1) {
        int M = 0;
        for (int i = 0; i < a.n_req; ++i) M = std::max(M, a.req[i].M);
        const int threads = a.G * M * (HD / 4);
        if (a.n_splits >= 4) hipLaunchKernelGGL((paged_merge_kernel<T, 4>), dim3((threads * 4 + 255) / 256, a.Hkv, a.n_req), dim3(256), 0, s, a);
        else hipLaunchKernelGGL((paged_merge_kernel<T, 1>), dim3((threads + 255) / 256, a.Hkv, a.n_req), dim3(256), 0, s, a);
    }
    return hipGetLastError();
}

// One pass of the shared form; rows beyond what a workgroup takes go to further row blocks.
template <typename T, int HD>
void launch_pass(const SharedArgs& a, int row_tiles, hipStream_t s) {
    const dim3 grid(a.n_splits, a.Hkv, a.n_req * a.row_blocks);
    if constexpr (sizeof(T) == 2) {
        if (row_tiles == 1) hipLaunchKernelGGL((paged_attn_kernel<T, HD, 1, 1, false, true>), grid, dim3(256), 0, s, a);
        else if (row_tiles == 2) hipLaunchKernelGGL((paged_attn_kernel<T, HD, 2, 1, false, true>), grid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL((paged_attn_kernel<T, HD, 2, 2, false, true>), grid, dim3(512), 0, s, a);
    } else {
        hipLaunchKernelGGL((paged_attn_kernel<T, HD, 1, 1, false, true>), grid, dim3(256), 0, s, a);
    }
}

template <typename T, int HD>
hipError_t launch_shared(const SharedPlan& p, hipStream_t s) {
    const SharedArgs& a = p.own;
    if (p.prefix.n_req) launch_pass<T, HD>(p.prefix, p.prefix_tiles, s);
    launch_pass<T, HD>(a, p.own_tiles, s);
    MergeGroups g{};
    int M = 0;
    for (int i = 0; i < p.prefix.n_req; ++i) {
        g.part0[i] = p.prefix.req[i].part0;
        g.splits[i] = p.prefix.req[i].splits;
    }
    for (int i = 0; i < a.n_req; ++i) M = std::max(M, a.req[i].M);
    const int threads = a.G * M * (HD / 4);
    if (p.places >= 4) hipLaunchKernelGGL((shared_merge_kernel<T, 4>), dim3((threads * 4 + 255) / 256, a.Hkv, a.n_req), dim3(256), 0, s, a, g);
    else hipLaunchKernelGGL((shared_merge_kernel<T, 1>), dim3((threads + 255) / 256, a.Hkv, a.n_req), dim3(256), 0, s, a, g);
    return hipGetLastError();
}

// Row tiles of a pass, its splits and its places from part0 on; at most `most_splits`.
int plan_pass(int dtype, SharedArgs& a, int part0, int most_splits) {
    int R = 0, most = 1;
    for (int i = 0; i < a.n_req; ++i) R = std::max(R, a.G * a.req[i].M);
    const int row_tiles = R <= 16 || dtype == 0 ? 1 : R <= 32 ? 2 : 4;
    a.tail_w = tail_weight(std::min(row_tiles, 2));
    a.row_blocks = (R + 16 * row_tiles - 1) / (16 * row_tiles);
    auto units = [&](const SharedReq& r) { return (r.n_paged + PAGE_TOK - 1) / PAGE_TOK - r.first + (r.L - r.n_paged + 63) / 64 * a.tail_w; };
    long long base = 0;
    for (int i = 0; i < a.n_req; ++i) {
        most = std::max(most, units(a.req[i]));
        base += (long long)a.Hkv * ((a.G * a.req[i].M + 16 * row_tiles - 1) / (16 * row_tiles));
    }
    const int n = std::min((int)std::min((long long)most_splits, std::max(1LL, TARGET_WGS / base)), (most + STREAMS - 1) / STREAMS);
    a.units_per_split = (most + n - 1) / n;
    a.n_splits = (most + a.units_per_split - 1) / a.units_per_split;
    for (int i = 0; i < a.n_req; ++i) {
        a.req[i].part0 = part0;
        a.req[i].splits = (units(a.req[i]) + a.units_per_split - 1) / a.units_per_split;
    }
    return row_tiles;
}

}  // namespace

int shared_max_places(int Hkv, long long R) { return 2 * paged_max_splits(Hkv, R); }

void shared_plan(int dtype, SharedPlan& p) {
    const int most = std::min(31, paged_max_splits(p.own.Hkv, (long long)p.own.G * p.own.rows));
    p.own.Rpad = (p.own.G * p.own.rows + 15) / 16 * 16;
    const int groups = p.prefix.n_req;
    (PagedBase&)p.prefix = (const PagedBase&)p.own;
    p.prefix.n_req = groups;
    p.prefix.n_splits = 0;
    if (groups) p.prefix_tiles = plan_pass(dtype, p.prefix, 0, most);
    p.own_tiles = plan_pass(dtype, p.own, p.prefix.n_splits, most);
    p.places = p.prefix.n_splits + p.own.n_splits;
}

hipError_t launch_shared_attention(int dtype, const SharedPlan& p, hipStream_t s) {
    if (dtype == 0) return p.own.hd == 64 ? launch_shared<float, 64>(p, s) : launch_shared<float, 128>(p, s);
    return p.own.hd == 64 ? launch_shared<bf16_t, 64>(p, s) : launch_shared<bf16_t, 128>(p, s);
}

int paged_max_splits(int Hkv, long long R) { return (int)std::min(64LL, std::max(1LL, TARGET_WGS / (Hkv * ((R + 63) / 64)))); }

int paged_plan(int dtype, PagedArgs& a) {
    int R = 0, most = 1;
    for (int i = 0; i < a.n_req; ++i) R = std::max(R, a.G * a.req[i].M);
    // (f32: twice the registers and LDS per row)
    const int row_tiles = R <= 16 || dtype == 0 ? 1 : R <= 32 ? 2 : 4;
    a.tail_w = tail_weight(std::min(row_tiles, 2));
    a.row_blocks = (R + 16 * row_tiles - 1) / (16 * row_tiles);
    long long base = 0;
    for (int i = 0; i < a.n_req; ++i) {
        most = std::max(most, units_of(a.req[i], a.tail_w));
        base += (long long)a.Hkv * ((a.G * a.req[i].M + 16 * row_tiles - 1) / (16 * row_tiles));
    }
    // one split length for all: finer splits for equal work of contexts of different lengths were no faster (32 tokens, 4 KV heads, 512 to 4096
    // slots: at most 2 splits 20.3 us, 3 or 4 22.5), as two short workgroups that meet on one unit take as long as a long one
    int n = std::min((int)std::min(64LL, std::max(1LL, TARGET_WGS / base)), (most + STREAMS - 1) / STREAMS);
    // Short contexts are not split: the waves' few more pages take no longer than a second, dependent launch (one row, us replayed: 32 heads, 1000 slots 9.7 ->
    // 8.0; 4 requests, 1500 15.6 -> 12.2; 8 KV heads, 8 requests, 1100 7.9 -> 6.5; 32 heads, 1500 10.5 -> 10.9, where the call gains 2; 2000 10.8 -> 13.0.
    // Two row tiles: 24 rows, 700 slots 11.6 -> 11.0, 28 rows, 1500 10.4 -> 13.6.  Four: 40 rows, 500 slots 15.2 -> 15.8).
    // f32, whose rounds of four pages take longer than the second launch from the second one on: one split against several, 4 heads of 64, 300 slots 8.5 us, 10.3;
    // 394 10.9, 10.7; 1000 16.4, 10.8; 32 heads of 128, 300 slots 13.8, 15.3; 394 18.9, 16.1; 1000 28.7, 16.4; 8 requests of 4 rows, 300 8.7, 10.6; 600 13.7, 11.3.
    if (most <= (dtype == 0 ? 6 : row_tiles == 1 ? 28 : row_tiles == 2 ? 20 : 0)) n = 1;
    a.units_per_split = (most + n - 1) / n;
    a.n_splits = (most + a.units_per_split - 1) / a.units_per_split;
    a.Rpad = (a.G * a.rows + 15) / 16 * 16;
    return row_tiles;
}

hipError_t launch_paged_attention(int dtype, const PagedArgs& a, int row_tiles, hipStream_t s) {
    if (dtype == 0) return a.hd == 64 ? launch<float, 64>(a, row_tiles, s) : launch<float, 128>(a, row_tiles, s);
    return a.hd == 64 ? launch<bf16_t, 64>(a, row_tiles, s) : launch<bf16_t, 128>(a, row_tiles, s);
}
