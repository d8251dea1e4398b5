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
#include <climits>

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
// PART: over what of the contexts a call goes: all of it; whole pages only, or what lies behind a page, whose sums are partial always; or all of it with the
// pages that a group shares named by the group's row of the table, in one split.
enum class Part { ALL, PAGES, REST, EACH };

// LDS of a workgroup, bytes: the waves' sums, or before that the staged values behind the pages; the workgroup's queries as fragments; the sums over the
// slots behind the pages, [wave][row][RROW], then (m, l).
template <typename T, int HD, int MTW, int RG, bool APART, Part PART>
struct PagedLds {
    static constexpr int PW = STREAMS * RG, TW = APART ? STREAMS : PW, RROW = HD + 4;
    static constexpr int STAGE = PART == Part::PAGES ? 0 : TW * RowTiles<T, HD, 1>::STAGE * (int)sizeof(T), RED = PW * 16 * (RROW + 2) * 4;
    static constexpr int SUMS = STAGE > RED ? STAGE : RED, Q = MTW * RG * RowTiles<T, HD, MTW>::NKT * 1024, TAIL = PART == Part::PAGES ? 16 : TW * 16 * (RROW + 2) * 4;
};

template <typename T, int HD, int MTW, int RG, bool APART, Part PART, typename Args, typename Req>
static __device__ __forceinline__ void paged_rows(const Args& a, const Req& rq, int split, int kvh, int rb, unsigned char* lds, unsigned char* q_lds, float* tail_o) {
    constexpr bool SHARED = PART == Part::PAGES || PART == Part::REST;
    constexpr int PW = STREAMS * RG, TW = APART ? STREAMS : PW;  // waves over pages, waves over the slots behind them
    constexpr int WAVES = APART ? PW + TW : PW;
    static_assert(!APART || RG == 1, "waves of one group");
    using RT = RowTiles<T, HD, MTW>;
    using frag_t = typename RT::frag_t;
    constexpr int NA = HD / 64, NHT = HD / 16, PER = RT::PER;
    constexpr int RROW = HD + 4;  // padded row of the sums that the waves exchange
    constexpr int WPR = STREAMS / MTW;  // waves that share a row tile behind the pages
    using TT = RowTiles<T, HD, 1>;
    constexpr int NKT = RT::NKT, QT = MTW * RG * NKT;  // fragments of the workgroup's queries

    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r16 = lane & 15, g = lane >> 4;
    const int M = rq.M, R = a.G * M, rho0 = rb * 16 * MTW * RG;
    if (rho0 >= R) return;  // a shorter request of the batch has no such row block
    const int L = rq.l_glo + rq.seg_off + M;
    int first_page = 0;  // (pages are counted from first_page on below)
    if constexpr (PART == Part::REST) first_page = rq.first;
    const int np = (rq.n_paged + PAGE_TOK - 1) / PAGE_TOK - first_page, nt = PART == Part::PAGES ? 0 : (L - rq.n_paged + 63) / 64;
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
    const bool tail = PART != Part::PAGES && j1 > j0;
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
        auto raw_id = [&](int t) __attribute__((always_inline)) {
            if constexpr (PART == Part::EACH) return (t < rq.first ? (cint_p)(a.table + (size_t)a.req[max(rq.group, 0)].seq * a.max_pages) : ids)[t];
            else return ids[t];
        };
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
        const long long first = k_tile(page_id(raw_id(t)));
        int ahead = raw_id(t + STREAMS < tp ? t + STREAMS : t);  // (in the loop's order, so that its waits can count)
        load_k(first);
        load_v(first + a.Hkv);
        for (; t < whole; t += STREAMS) {
            // behind the wave's last tile the same one is fetched once more, from the caches: no load hangs on a branch
            const long long next = k_tile(page_id(ahead));
            ahead = raw_id(t + 2 * STREAMS < tp ? t + 2 * STREAMS : t);
            scores();
            load_k(next);
#pragma unroll
            for (int i = 0; i < MTW; ++i) rt.template softmax<4, false>(i, st[i], a.scale_log2, 0ull);
            products();
            load_v(next + a.Hkv);
        }
        if (PART != Part::PAGES && t < tp) {  // the partial page
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
                if constexpr (SHARED) prow = ((size_t)((PART == Part::REST ? a.own_place : 0) + split) * a.Hkv + kvh) * a.Rpad + (size_t)(rho / M) * a.rows + rq.row0 + rho % M;
                else prow = ((size_t)split * a.Hkv + kvh) * a.Rpad + (size_t)a.G * rq.row0 + rho;
                *(f32x4*)(a.part_o + prow * HD + c) = o;
                if (c == 0) *(float2*)(a.part_ml + prow * 2) = make_float2(mm, den);
            }
        }
    }
}

template <typename T, int HD, int MTW, int RG, bool APART>
__global__ void __launch_bounds__(sizeof(T) == 2 ? 512 : 256) paged_attn_kernel(const PagedArgs a) {
    using Lds = PagedLds<T, HD, MTW, RG, APART, Part::ALL>;
    __shared__ __align__(16) unsigned char lds[Lds::SUMS];
    __shared__ __align__(16) unsigned char q_lds[Lds::Q];
    __shared__ __align__(16) float tail_o[Lds::TAIL / 4];
    const PagedReq rq = a.req[blockIdx.z / a.row_blocks];
    paged_rows<T, HD, MTW, RG, APART, Part::ALL>(a, rq, blockIdx.x, blockIdx.y, blockIdx.z % a.row_blocks, lds, q_lds, tail_o);
}

// Whole shared pages under 32 rows, 16 bits, by 32x32x16 products: S^T = K . Q^T and O^T += V^T . P^T with query row l % 32 in lane l.
// As above a wave takes every fourth page by itself, codes from memory to registers and from there to operands; nothing is in LDS until the sums meet.  Lane
// l's 16 codes of token l % 32 are columns 32 j + 16 (l / 32) on, so the queries' columns are taken in that order too.
//
// Bound: neither side alone.  Called back to back, 110 us over 16384 shared slots (8 requests of 32 rows, 32 heads of 128: 69.3 GFLOP, 137 MB) are 81 without
// the loads of pages, 76 without the matrix products and 105 without the exponentials.  Other ways to the same end, the launch over these shared pages alone: the
// 16x16x32 products of the kernel above 89 us, this one 85; codes expanded once for 128 rows into LDS 84, or with one half of the waves at their products
// while the other expands and takes exponentials 80, but 21.7 where 4096 slots are shared (16 requests, 28/4 heads), against 19.6; 64 rows to a wave 121.
typedef float f32x16 __attribute__((ext_vector_type(16)));

static __device__ __forceinline__ float half_max(float x) {  // of a lane's value and that of the lane 32 away
    typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
    const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

template <int HD>
struct PagesLds {
    static constexpr int RROW = HD + 4, SUMS = STREAMS * 32 * (RROW + 2) * 4;
};
template <int HD>
static __device__ __forceinline__ void shared_pages(const SharedArgs& a, const SharedReq& rq, int split, int kvh, int rb, unsigned char* lds) {
    using E = Elem<bf16_t>;
    constexpr int NJ = HD / 32, NHT = HD / 32, RROW = PagesLds<HD>::RROW;
    constexpr float HEADROOM = RowTiles<bf16_t, HD, 1>::HEADROOM;
    float* ro = (float*)lds;                             // the waves' sums: [wave][row][RROW]
    float2* rml = (float2*)(ro + STREAMS * 32 * RROW);     // [wave][row]
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), c32 = lane & 31, h = lane >> 5;
    const int M = rq.M, R = a.G * M, blk0 = rb * 32;
    const int np = rq.n_paged / PAGE_TOK, t0 = split * a.units_per_split, tp = min(np, t0 + a.units_per_split);
    const int rho = blk0 + c32;
    const bool ok = rho < R;
    f32x16 acc[NHT];
#pragma unroll
    for (int k = 0; k < NHT; ++k)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[k][v] = 0.f;
    float m = FS_NEG_INF, ms = 0.f, l = 0.f;  // ms: what is subtracted, m where that is finite
    bool bad = false;
    if (t0 + w < tp) {
        // ids and scales by scalar loads: they do not stand in the way of the waits for codes (nothing writes them while the kernel runs)
        typedef const __attribute__((address_space(4))) int32_t* cint_p;
        typedef const __attribute__((address_space(4))) float* cfloat_p;
        const cint_p ids = (cint_p)(a.table + (size_t)rq.seq * a.max_pages);
        const cfloat_p scales = (cfloat_p)a.scales;
        u32x4 kc[2][NJ], vc[NHT][2];
        float ks, vs;
        // an id outside the pool: page 0 is read in its place and the rows become NaN
        auto tile_of = [&](int raw) __attribute__((always_inline)) {
            const int id = __builtin_amdgcn_readfirstlane(raw);
            const bool in = (unsigned)id < (unsigned)a.n_pages;
            bad |= !in;
            return (long long)(in ? id : 0) * a.page_tiles + a.tile0 + kvh;
        };
        const unsigned off = c32 * 64 + h * 16;
        auto load_k = [&](long long tile, int j) __attribute__((always_inline)) {
            const unsigned char* p = a.codes + tile * (PAGE_TOK * HD);
#pragma unroll
            for (int s = 0; s < 2; ++s) kc[s][j] = *(const u32x4*)(p + (off + (j / 2 * 4096 + s * 2048 + j % 2 * 32)));
        };
        auto load_v = [&](long long tile, int k) __attribute__((always_inline)) {
            const unsigned char* p = a.codes + (tile + a.Hkv) * (PAGE_TOK * HD);
#pragma unroll
            for (int x = 0; x < 2; ++x) vc[k][x] = *(const u32x4*)(p + (off + (k * 2048 + x * 32)));
        };
        int t = t0 + w;
        long long tile = tile_of(ids[t]);
        int ahead = ids[min(t + STREAMS, tp - 1)];
#pragma unroll
        for (int j = 0; j < NJ; ++j) load_k(tile, j);
#pragma unroll
        for (int k = 0; k < NHT; ++k) load_v(tile, k);
        ks = scales[tile];
        vs = scales[tile + a.Hkv];
        bf16x8 qf[NJ][2];  // columns 32 j + 16 h + 8 x on: the order in which a lane has 16 codes of a token
        {
            const int rr = ok ? rho : 0;
            const bf16_t* qp = (const bf16_t*)a.q + (size_t)(rq.row0 + rr % M) * a.ldq + (size_t)(kvh * a.G + rr / M) * HD + h * 16;
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int x = 0; x < 2; ++x) qf[j][x] = ok ? *(const bf16x8*)(qp + j * 32 + x * 8) : E::zero();
        }
        for (; t < tp; t += STREAMS) {
            // behind the wave's last tile one is fetched once more, from the caches: no load hangs on a branch
            const long long next = tile_of(ahead);
            ahead = ids[min(t + 2 * STREAMS, tp - 1)];
            const float ks1 = scales[next], vs1 = scales[next + a.Hkv];
            f32x16 st[2];
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int v = 0; v < 16; ++v) st[s][v] = 0.f;
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        const unsigned wd[2] = {kc[s][j][2 * x], kc[s][j][2 * x + 1]};
                        st[s] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(Codes<bf16_t>::frag(wd, ks), qf[j][x], st[s], 0, 0, 0);
                    }
                load_k(next, j);  // (the registers are free: the next page's codes have most of an iteration to come)
                __builtin_amdgcn_sched_barrier(0);
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
                for (int k = 0; k < NHT; ++k)
#pragma unroll
                    for (int v = 0; v < 16; ++v) acc[k][v] *= alpha;
                m = mnew;
            }
            float sum[2] = {0.f, 0.f};
            bf16x8 pf[4];
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(st[c / 2][(c % 2) * 8 + e], a.scale_log2, -ms));
                    pf[c][e] = (bf16_t)x;  // (half a step of 2^-8 of a probability, of the size of the result's own rounding; the sum is of the unrounded)
                    sum[e & 1] += x;
                }
            l += sum[0] + sum[1];
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int k = 0; k < NHT; ++k) {
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const unsigned wd[2] = {vc[k][0][c], vc[k][1][c]};
                    acc[k] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(Codes<bf16_t>::frag(wd, vs), pf[c], acc[k], 0, 0, 0);
                }
                load_v(next, k);
                __builtin_amdgcn_sched_barrier(0);
            }
            ks = ks1;
            vs = vs1;
        }
    }
    // the streams' sums
    l += __shfl_xor(l, 32, FS_WAVE);
    if (bad) l = __builtin_nanf("");
#pragma unroll
    for (int k = 0; k < NHT; ++k)
#pragma unroll
        for (int v = 0; v < 16; v += 4)
            *(f32x4*)(ro + (w * 32 + c32) * RROW + k * 32 + 2 * v + 4 * h) = f32x4{acc[k][v], acc[k][v + 1], acc[k][v + 2], acc[k][v + 3]};
    if (h == 0) rml[w * 32 + c32] = make_float2(m, l);
    __syncthreads();
    constexpr int LPR = HD / 4, STEP = 64 * STREAMS / LPR;  // lanes to a row, rows at a time
    const int c = tid % LPR * 4;
#pragma unroll
    for (int r = tid / LPR; r < 32; r += STEP) {
        const int row = blk0 + r;
        if (row >= R) break;
        float2 ml[STREAMS];
        float mm = FS_NEG_INF;
#pragma unroll
        for (int k = 0; k < STREAMS; ++k) {
            ml[k] = rml[k * 32 + r];
            mm = fmaxf(mm, ml[k].x);
        }
        const float msub = mm == FS_NEG_INF ? 0.f : mm;
        float den = 0.f;
        f32x4 o{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < STREAMS; ++k) {
            const float wt = __builtin_amdgcn_exp2f(ml[k].x - msub);
            den += wt * ml[k].y;
            o += *(const f32x4*)(ro + (k * 32 + r) * RROW + c) * wt;
        }
        const size_t prow = ((size_t)split * a.Hkv + kvh) * a.Rpad + (size_t)(row / M) * a.rows + rq.row0 + row % M;
        *(f32x4*)(a.part_o + prow * HD + c) = o;
        if (c == 0) *(float2*)(a.part_ml + prow * 2) = make_float2(mm, den);
    }
}

// Requests whose contexts begin alike: sums over what is shared and over what follows are partial softmax sums like those of splits, and are joined as these
// are.  The pages that a group shares are read once for the stacked rows of all its requests, not once for each: 32 tokens behind 2048 shared slots
// (32 heads of 128) read 17 MB of them, not 537.  The groups' stacked rows over those pages (PT tiles of 16 to a workgroup) and the requests' rows
// over what follows (OT) are one launch, the groups first, so that the short ones fill the gaps (as two launches: 32 tokens 29.8 us a call, as one
// 23.1; 16 trees, 28/4 heads, 4096 shared 34.1 and 22.9; two prompts 37.5 and 30.7).  A workgroup is number id - wg0 of its entry, KV head by KV head,
// then by row block, then by split.
template <typename T, int HD, int PT, int OT>
__global__ void __launch_bounds__(sizeof(T) == 2 ? 512 : 256) shared_attn_kernel(const SharedArgs a) {
    using P = PagedLds<T, HD, 1, 1, false, Part::PAGES>;
    using O = PagedLds<T, HD, OT, 1, false, Part::REST>;
    constexpr int NP = PT == 1 ? P::SUMS + P::Q + P::TAIL : PagesLds<HD>::SUMS, NO = O::SUMS + O::Q + O::TAIL;
    __shared__ __align__(16) unsigned char lds[NP > NO ? NP : NO];
    static_assert(2 * PAGED_MAX_REQ == FS_WAVE, "a lane for each entry");
    const int lane = threadIdx.x & 63, id = blockIdx.x;
    const int e = __builtin_amdgcn_readfirstlane(__popcll(__ballot(a.wg0[lane] <= id)) - 1);  // (entries that are not there begin behind the last workgroup)
    const int at = id - a.wg0[e], kvh = at % a.Hkv, block = at / a.Hkv;
    const bool prefix = e < a.n_prefix;
    const SharedReq rq = a.req[e];
    const int tiles = 16 * (prefix ? PT : OT), blocks = (a.G * rq.M + tiles - 1) / tiles;
    const int rb = block % blocks, split = block / blocks;
    if (prefix) {
        if constexpr (PT == 1) paged_rows<T, HD, 1, 1, false, Part::PAGES>(a, rq, split, kvh, rb, lds, lds + P::SUMS, (float*)(lds + P::SUMS + P::Q));
        else shared_pages<HD>(a, rq, split, kvh, rb, lds);
        return;
    }
    paged_rows<T, HD, OT, 1, false, Part::REST>(a, rq, split, kvh, rb, lds, lds + O::SUMS, (float*)(lds + O::SUMS + O::Q));
}

// Requests whose contexts begin alike, each by itself: see shared_plan.
template <typename T, int HD, int OT, bool APART>
__global__ void __launch_bounds__(sizeof(T) == 2 ? 512 : 256) shared_each_kernel(const SharedArgs a) {
    using Lds = PagedLds<T, HD, OT, 1, APART, Part::EACH>;
    __shared__ __align__(16) unsigned char lds[Lds::SUMS];
    __shared__ __align__(16) unsigned char q_lds[Lds::Q];
    __shared__ __align__(16) float tail_o[Lds::TAIL / 4];
    const SharedReq rq = a.req[a.n_prefix + blockIdx.z];
    paged_rows<T, HD, OT, 1, APART, Part::EACH>(a, rq, 0, blockIdx.x, blockIdx.y, lds, q_lds, tail_o);
}

// out = sum_s 2^(m_s - m) O_s / sum_s 2^(m_s - m) l_s.  LANES adjacent lanes share four columns of a row and take splits q, q + LANES, ...,
// then meet pairwise in a fixed order.  (Its sums are written out here: by merge_in and merge_lanes below the compiler fuses other products of them, and results
// that were there before would differ in their last bit.)
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
        const float mn = fmaxf(m, ml.x), ms = mn == FS_NEG_INF ? 0.f : mn;
        const float w0 = __builtin_amdgcn_exp2f(m - ms), w1 = __builtin_amdgcn_exp2f(ml.x - ms);
        den = den * w0 + ml.y * w1;
        o = o * w0 + v * w1;
        m = mn;
    }
#pragma unroll
    for (int x = 1; x < LANES; x <<= 1) {
        const float m2 = __shfl_xor(m, x, FS_WAVE), den2 = __shfl_xor(den, x, FS_WAVE);
        f32x4 o2;
#pragma unroll
        for (int e = 0; e < 4; ++e) o2[e] = __shfl_xor(o[e], x, FS_WAVE);
        const float mn = fmaxf(m, m2), ms = mn == FS_NEG_INF ? 0.f : mn;
        const float w1 = __builtin_amdgcn_exp2f(m - ms), w2 = __builtin_amdgcn_exp2f(m2 - ms);
        den = den * w1 + den2 * w2;  // lane 0 of a group, whose sum is stored, always adds the higher lane's term second
        o = o * w1 + o2 * w2;
        m = mn;
    }
    if (q != 0) return;
    store_row<T>(a, rq, kvh, loc, c, o, den);
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

// The same over a row's places: those of its group, then its own.
template <typename T, int LANES>
__global__ void __launch_bounds__(256) shared_merge_kernel(const SharedArgs a) {
    const SharedReq rq = a.req[a.n_prefix + blockIdx.z];
    const int chunks = a.hd / 4, id = (blockIdx.x * 256 + threadIdx.x) / LANES, q = threadIdx.x % LANES;
    const int kvh = blockIdx.y, loc = id / chunks, c = id % chunks * 4;
    if (loc >= a.G * rq.M) return;
    const int gn = rq.group < 0 ? 0 : a.req[rq.group].splits, all = gn + rq.splits;
    const size_t step = (size_t)a.Hkv * a.Rpad, row = (size_t)kvh * a.Rpad + (size_t)(loc / rq.M) * a.rows + rq.row0 + loc % rq.M;
    float m = FS_NEG_INF, den = 0.f;
    f32x4 o{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = q; s < all; s += LANES) {
        const size_t at = row + (size_t)(s < gn ? s : a.own_place + s - gn) * step;
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
        if (row_tiles == 1 && apart) hipLaunchKernelGGL((paged_attn_kernel<T, HD, 1, 1, true>), grid, dim3(512), 0, s, a);
        else if (row_tiles == 1) hipLaunchKernelGGL((paged_attn_kernel<T, HD, 1, 1, false>), grid, dim3(256), 0, s, a);
        else if (row_tiles == 2 && apart) hipLaunchKernelGGL((paged_attn_kernel<T, HD, 2, 1, true>), grid, dim3(512), 0, s, a);
        else if (row_tiles == 2) hipLaunchKernelGGL((paged_attn_kernel<T, HD, 2, 1, false>), grid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL((paged_attn_kernel<T, HD, 2, 2, false>), grid, dim3(512), 0, s, a);
    } else {
        hipLaunchKernelGGL((paged_attn_kernel<T, HD, 1, 1, false>), grid, dim3(256), 0, s, a);
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

template <typename T, int HD>
hipError_t launch_shared(const SharedPlan& p, hipStream_t s) {
    const SharedArgs& a = p.a;
    if (p.each) {
        const dim3 grid(a.Hkv, a.row_blocks, a.n_req);
        if constexpr (sizeof(T) == 2) {
            if (p.own_tiles == 2) hipLaunchKernelGGL((shared_each_kernel<T, HD, 2, true>), grid, dim3(512), 0, s, a);
            else hipLaunchKernelGGL((shared_each_kernel<T, HD, 1, true>), grid, dim3(512), 0, s, a);
        } else {
            hipLaunchKernelGGL((shared_each_kernel<T, HD, 1, false>), grid, dim3(256), 0, s, a);
        }
        return hipGetLastError();
    }
    const dim3 grid(p.wgs);
    if constexpr (sizeof(T) == 2) {
        if (p.own_tiles == 2) hipLaunchKernelGGL((shared_attn_kernel<T, HD, 2, 2>), grid, dim3(256), 0, s, a);
        else if (p.prefix_tiles == 2) hipLaunchKernelGGL((shared_attn_kernel<T, HD, 2, 1>), grid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL((shared_attn_kernel<T, HD, 1, 1>), grid, dim3(256), 0, s, a);
    } else {
        hipLaunchKernelGGL((shared_attn_kernel<T, HD, 1, 1>), grid, dim3(256), 0, s, a);
    }
    int M = 0;
    for (int i = 0; i < a.n_req; ++i) M = std::max(M, a.req[a.n_prefix + i].M);
    const int threads = a.G * M * (HD / 4);
    if (p.places >= 4) hipLaunchKernelGGL((shared_merge_kernel<T, 4>), dim3((threads * 4 + 255) / 256, a.Hkv, a.n_req), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((shared_merge_kernel<T, 1>), dim3((threads + 255) / 256, a.Hkv, a.n_req), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace

int shared_max_places(int Hkv, long long R) { return std::max(2 * std::min(31, paged_max_splits(Hkv, R)), paged_max_splits(Hkv, R)); }  // (without groups: the paged attention's)

// What a workgroup costs besides its pages, in pages: queries, the first page's way from memory, sums (6 us, a round of four pages 2.6, of 64 rows; what it
// leads to for 32 is in shared_plan).
constexpr int WG_UNITS = 9;
// Workgroups up to which short contexts are taken each by itself: one to a compute unit, a single round (us a call, each by itself and shared: 3 tokens, f32, 128
// shared slots 9.2, 12.2; 28/4 heads, 32 tokens, 512 shared 9.3, 12.5; 32 heads, 8 tokens, 1024 9.7, 12.3, 2 tokens, 1536 10.7, 12.0; with more workgroups, replayed
// from a graph: 16 tokens, 512 18.3, 17.1; 32 tokens, 256 28.9, 23.4).
constexpr int EACH_WGS = TARGET_WGS;

void shared_plan(int dtype, SharedPlan& p) {
    SharedArgs& a = p.a;
    const int entries = a.n_prefix + a.n_req;
    int R[2] = {0, 0};  // most stacked rows of an entry: groups, requests
    for (int e = 0; e < entries; ++e) R[e >= a.n_prefix] = std::max(R[e >= a.n_prefix], a.G * a.req[e].M);
    // 32 rows at most to a workgroup of four waves, two on a compute unit: 64 rows in eight waves, of which two read the same page, leave a unit to one workgroup
    // and its gaps to nobody (us a call, 64 rows and 32, medians: two prompts 31.0, 27.9; 8 trees of 16384 88.4, 84.6; 12 segments of 16 rows behind 1024
    // 20.4, 18.5; 16 trees, 28/4 heads, 4096 shared 24.8, 24.6).
    auto tiles_of = [&](int rows) { return rows <= 16 || dtype == 0 ? 1 : 2; };
    p.own_tiles = tiles_of(R[1]);
    p.prefix_tiles = std::max(p.own_tiles, tiles_of(R[0]));
    a.tail_w = tail_weight(std::min(p.own_tiles, 2));
    a.Rpad = (a.G * a.rows + 15) / 16 * 16;
    // Pages (tiles behind them weighed as such) and workgroups of an entry that is not split.
    int units[2 * PAGED_MAX_REQ], longest = 1, own = 1;
    long long base[2 * PAGED_MAX_REQ], work = 0;
    for (int e = 0; e < entries; ++e) {
        const SharedReq& r = a.req[e];
        const int rows = 16 * (e < a.n_prefix ? p.prefix_tiles : p.own_tiles);
        units[e] = (r.n_paged + PAGE_TOK - 1) / PAGE_TOK - r.first;
        if (e >= a.n_prefix) units[e] += (r.l_glo + r.seg_off + r.M - r.n_paged + 63) / 64 * a.tail_w;
        base[e] = (long long)a.Hkv * ((a.G * r.M + rows - 1) / rows);
        longest = std::max(longest, units[e]);
        if (e >= a.n_prefix) own = std::max(own, units[e]);
        work += base[e] * units[e];
    }
    // Short contexts of few requests: every request by itself, in one launch, as the paged attention takes them, and no longer than it takes in one split.
    int whole = 0;
    long long each = 0;
    for (int e = a.n_prefix; e < entries; ++e) {
        whole = std::max(whole, units[e] + a.req[e].first);
        each += base[e];
    }
    p.each = each <= EACH_WGS && whole <= (dtype == 0 ? 6 : p.own_tiles == 1 ? 28 : 20);
    if (p.each) {
        a.n_splits = 1;
        a.units_per_split = 1 << 24;
        a.row_blocks = (R[1] + 16 * p.own_tiles - 1) / (16 * p.own_tiles);
        p.places = 2;
        p.wgs = each;
        return;
    }
    // One length of splits for all: the number of the longest entry's that lets the launch end first, by the longest workgroup, or by what each of the
    // places for workgroups has to do and, where a second round starts, half of a late workgroup.  Splits of the longest entry, us a call, medians: 16 trees,
    // 28/4 heads, 4096 shared: 1 26.8, 2 23.9, 3 (taken) 25.2, 4 29.2; 8 trees of 16384: 1 87.7, 2 (taken, the most) 84.6; 4 tokens behind 8192: 1 40.9,
    // 2 25.2, 4 18.9, 8 (taken, the most) 18.8; 32 tokens behind 2048: 1 22.9, 2 (taken) 23.2, 4 25.2; 12 segments of 16 rows behind 1024: 1 (taken) 18.7, 2 21.1.
    const int most = std::min({31, paged_max_splits(a.Hkv, (long long)a.G * a.rows), (longest + STREAMS - 1) / STREAMS});
    const int places = 2 * TARGET_WGS;
    long long best = -1;
    for (int n = 1; n <= most; ++n) {
        const int u = (longest + n - 1) / n;
        long long wgs = 0;
        for (int e = 0; e < entries; ++e) wgs += base[e] * ((units[e] + u - 1) / u);
        const long long load = (work + wgs * WG_UNITS) / places, cost = std::max((long long)u + WG_UNITS, wgs > places ? load + (std::min(own, u) + WG_UNITS) / 2 : load);
        if (best < 0 || cost < best) {
            best = cost;
            a.units_per_split = u;
        }
    }
    int splits[2] = {0, 0};
    long long at = 0;
    for (int e = 0; e < entries; ++e) {
        a.wg0[e] = (int)std::min(at, (long long)INT_MAX);
        a.req[e].splits = (units[e] + a.units_per_split - 1) / a.units_per_split;
        splits[e >= a.n_prefix] = std::max(splits[e >= a.n_prefix], a.req[e].splits);
        at += base[e] * a.req[e].splits;
    }
    for (int e = entries; e < 2 * PAGED_MAX_REQ; ++e) a.wg0[e] = INT_MAX;
    p.wgs = at;
    a.own_place = splits[0];
    p.places = splits[0] + splits[1];
}

hipError_t launch_shared_attention(int dtype, const SharedPlan& p, hipStream_t s) {
    if (dtype == 0) return p.a.hd == 64 ? launch_shared<float, 64>(p, s) : launch_shared<float, 128>(p, s);
    return p.a.hd == 64 ? launch_shared<bf16_t, 64>(p, s) : launch_shared<bf16_t, 128>(p, s);
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
