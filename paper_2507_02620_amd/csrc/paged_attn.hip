// Attention of draft-tree segments against a context whose settled tokens lie in pages of 64, 8 bits each (e4m3, a power-of-two scale
// per page, K or V, head), and whose newest slots lie in the 16- or 32-bit cache.
//
// The rows of the G query heads that share a KV head are stacked (R = G * M), as in the tree-attention kernel.  Grid: (split, KV head,
// request x row block); a workgroup's four waves hold the same 16 * MTW rows and take alternate tiles of 64 slots, so nothing is
// shared until the end and no wave waits for another: a page is stored in matrix-operand order, every lane loads its 16 codes of
// a fragment pair straight into registers (1 KiB per wave and load) and one instruction turns two codes into two bf16 values, times
// the scale, exactly (4 significant bits, a power of two).  What is multiplied is what the page stands for; nothing is rounded.
// The waves' sums meet in LDS, those of the splits in paged_merge_kernel, both in a fixed order.
//
// Bound: the stream of the pages (1 byte per element, half of what a 16-bit cache takes).
#include "paged.hpp"
#include "rows_attn.hpp"

#include <algorithm>
#include <type_traits>

namespace {

constexpr int WAVES = 4;

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
static __device__ __forceinline__ bool sees_nothing(const PagedArgs& a, const PagedReq& rq, int row) {
    if (rq.l_glo > 0 || !a.anc) return false;
    const int T = rq.seg_off + rq.M;
    const uint64_t* w = a.anc + (size_t)row * FS_ANC_WORDS;
    for (int i = 0; i * 64 < T; ++i) {
        const int left = T - i * 64;
        if (w[i] & (left >= 64 ? ~0ull : (1ull << left) - 1)) return false;
    }
    return true;
}

template <typename T>
static __device__ __forceinline__ void store_row(const PagedArgs& a, const PagedReq& rq, int kvh, int loc, int c, const f32x4& o, float den) {
    using E = Elem<T>;
    const int row = rq.row0 + loc % rq.M, qh = kvh * a.G + loc / rq.M;
    float inv = 1.0f / den;
    f32x4 v = o * inv;
    if (den == 0.f && sees_nothing(a, rq, row)) v = f32x4{0.f, 0.f, 0.f, 0.f};
    T* p = a.ldo ? (T*)a.o + (size_t)row * a.ldo + (size_t)qh * a.hd + c
                 : (T*)a.o + frag_major_index<T>(row, qh * a.hd + c, a.Hq * a.hd / E::KT);
    *(typename E::out4_t*)p = E::pack4(v[0], v[1], v[2], v[3]);
}

template <typename T, int HD, int MTW>
__global__ void __launch_bounds__(WAVES * 64) __attribute__((amdgpu_waves_per_eu(1))) paged_attn_kernel(const PagedArgs a) {
    using RT = RowTiles<T, HD, MTW>;
    using frag_t = typename RT::frag_t;
    constexpr int NA = HD / 64, NHT = HD / 16, PER = RT::PER;
    constexpr int RROW = HD + 4;  // padded row of the sums that the waves exchange
    constexpr int LDS_STAGE = WAVES * RT::STAGE * (int)sizeof(T), LDS_RED = WAVES * 16 * (RROW + 2) * 4;
    __shared__ __align__(16) unsigned char lds[LDS_STAGE > LDS_RED ? LDS_STAGE : LDS_RED];

    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r16 = lane & 15, g = lane >> 4;
    const int split = blockIdx.x, kvh = blockIdx.y, rqi = blockIdx.z / a.row_blocks, rb = blockIdx.z % a.row_blocks;
    const PagedReq rq = a.req[rqi];
    const int M = rq.M, R = a.G * M, rho0 = rb * 16 * MTW;
    if (rho0 >= R) return;  // a shorter request of the batch has no such row block
    const int L = rq.l_glo + rq.seg_off + M;
    const int np = (rq.n_paged + PAGE_TOK - 1) / PAGE_TOK, nt = (L - rq.n_paged + 63) / 64, tiles = np + nt;
    const int t0 = split * a.tiles_per_split, t1 = min(tiles, t0 + a.tiles_per_split);

    RT rt;
    rt.init();
    int seg_r[MTW];
    bool rok[MTW];
#pragma unroll
    for (int i = 0; i < MTW; ++i) {
        const int rho = rho0 + i * 16 + r16;
        rok[i] = rho < R;
        const int rr = rok[i] ? rho : 0;
        seg_r[i] = rr % M;
        rt.load_q(i, (const T*)a.q + (size_t)(rq.row0 + seg_r[i]) * a.ldq + (size_t)(kvh * a.G + rr / M) * HD, rok[i], g);
    }

    // ---- settled pages: the wave's tiles t0 + w, + 4, ...; the next one's K and V codes are on their way while one is computed ----
    bool bad = false;
    const int tp = min(t1, np);
    if (t0 + w < tp) {
        const int32_t* ids = a.table + (size_t)rq.seq * a.max_pages;
        const int lane16 = r16 * 4 + g;  // the lane's 16 bytes of a KiB in operand order
        u32x4 kc[4][NA], vc[NHT];
        float ks, vs, kn, vn;
        // an id outside the pool: page 0 is read in its place and the rows become NaN
        auto page_id = [&](int raw) {
            const int id = __builtin_amdgcn_readfirstlane(raw);
            const bool ok = (unsigned)id < (unsigned)a.n_pages;
            bad |= !ok;
            return ok ? id : 0;
        };
        auto k_tile = [&](int id) { return (long long)id * a.page_tiles + a.tile0 + kvh; };
        auto load_k = [&](long long tile) {
            const u32x4* p = (const u32x4*)(a.codes + tile * (PAGE_TOK * HD)) + lane16;
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int c = 0; c < NA; ++c) kc[j][c] = *(p + c * 256 + j * 64);
            kn = a.scales[tile];
        };
        auto load_v = [&](long long tile) {
            const u32x4* p = (const u32x4*)(a.codes + tile * (PAGE_TOK * HD)) + lane16;
#pragma unroll
            for (int n = 0; n < NHT; ++n) vc[n] = *(p + n * 64);
            vn = a.scales[tile];
        };
        auto step = [&](int t, long long next, auto more_tag) __attribute__((always_inline)) {
            constexpr bool MORE = decltype(more_tag)::value;
            ks = kn;
            f32x4 st[MTW][4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
#pragma unroll
                for (int i = 0; i < MTW; ++i) st[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < NA; ++c) {
                    const unsigned wd[4] = {kc[j][c][0], kc[j][c][1], kc[j][c][2], kc[j][c][3]};
#pragma unroll
                    for (int h = 0; h < PER; ++h) {
                        const frag_t kf = Codes<T>::frag(wd + h * (4 / PER), ks);
#pragma unroll
                        for (int i = 0; i < MTW; ++i) st[i][j] = RT::E::mma(kf, rt.qf[i][c * PER + h], st[i][j]);
                    }
                }
            }
            if (MORE) load_k(next);
            // only the last page of a context can be partial, and no tile follows it
            const int cnt = MORE ? 0 : rq.n_paged - t * PAGE_TOK;
            if (!MORE && cnt < PAGE_TOK) {
                const unsigned long long vis = ((1ull << cnt) - 1) >> (g * 4);
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
            } else {
#pragma unroll
                for (int i = 0; i < MTW; ++i) rt.template softmax<4, false>(i, st[i], a.scale_log2, 0ull);
            }
            vs = vn;
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
                }
            }
            if (MORE) load_v(next + a.Hkv);
        };
        int t = t0 + w;
        const long long first = k_tile(page_id(ids[t]));
        load_k(first);
        load_v(first + a.Hkv);
        int ahead = ids[min(t + WAVES, np - 1)];
        for (; t + WAVES < tp; t += WAVES) {
            const long long next = k_tile(page_id(ahead));
            ahead = ids[min(t + 2 * WAVES, np - 1)];
            step(t, next, std::integral_constant<bool, true>{});
        }
        step(t, 0, std::integral_constant<bool, false>{});
    }

    // ---- slots behind them, in the cache: halves of 32, masked where they hold draft slots ----
    {
        const T* kbase = (const T*)rq.tail + a.layer_off + (size_t)kvh * a.stride_head;
        T* vt = (T*)lds + w * RT::STAGE;
        // (the wave's first tile of the split behind the pages)
        int t = t0 + w;
        if (t < np) t += (np - t + WAVES - 1) / WAVES * WAVES;
        for (; t < t1; t += WAVES)
#pragma nounroll
            for (int h = 0; h < 2; ++h) {
                const int s0 = rq.n_paged + (t - np) * 64 + h * 32;
                if (s0 >= L) break;
                const int valid = min(L - s0, 32), d0 = s0 - rq.l_glo;
                const unsigned in = valid == 32 ? ~0u : (1u << valid) - 1;
                unsigned vis[MTW];
                bool any = false, part = false;
#pragma unroll
                for (int i = 0; i < MTW; ++i) {
                    unsigned m = ~0u;
                    if (d0 + 32 > 0) {  // some of the slots are draft slots: slot s0 + b is S index d0 + b
                        if (a.anc) {
                            const uint64_t* am = a.anc + (size_t)(rq.row0 + seg_r[i]) * FS_ANC_WORDS;
                            if (d0 >= 0) {
                                const int wd = d0 >> 6, sh = d0 & 63;
                                uint64_t x = am[wd] >> sh;
                                if (sh > 32 && wd + 1 < FS_ANC_WORDS) x |= am[wd + 1] << (64 - sh);
                                m = (unsigned)x;
                            } else {
                                m = (unsigned)(((1ull << -d0) - 1) | (am[0] << -d0));
                            }
                        } else {
                            const int n = rq.seg_off + seg_r[i] + 1 - d0;  // a chain: S indices up to the row's own
                            m = n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1;
                        }
                    }
                    m = rok[i] ? m & in : 0u;
                    vis[i] = m;
                    any |= m != 0;
                    part |= rok[i] && m != ~0u;
                }
                if (__ballot(any) == 0) continue;
                const T* kp = kbase + (long long)(s0 - rq.n_paged) * a.stride_tok;
                if (__ballot(part) != 0) rt.template half<true>(kp, kp + a.stride_kv, a.stride_tok, a.stride_tok, valid - 1, vis, a.scale_log2, vt, lane);
                else rt.template half<false>(kp, kp + a.stride_kv, a.stride_tok, a.stride_tok, valid - 1, vis, a.scale_log2, vt, lane);
            }
    }

    // ---- the waves' sums: one row tile at a time through LDS ----
    float* ro = (float*)lds;                       // [wave][row][RROW]
    float* rml = ro + WAVES * 16 * RROW;           // [wave][row][2]
#pragma unroll
    for (int i = 0; i < MTW; ++i) {
        if (rho0 + i * 16 >= R) break;  // uniform
        __syncthreads();
        const float l = bad ? __builtin_nanf("") : rt.row_sum(i);
#pragma unroll
        for (int n = 0; n < NHT; ++n) *(f32x4*)(ro + (w * 16 + r16) * RROW + n * 16 + g * 4) = rt.acc[i][n];
        if (g == 0) *(float2*)(rml + (w * 16 + r16) * 2) = make_float2(rt.m[i], l);
        __syncthreads();
        const int row = tid >> 4, rho = rho0 + i * 16 + row;
        if (rho >= R) continue;
        float2 ml[WAVES];
        float mm = FS_NEG_INF;
#pragma unroll
        for (int k = 0; k < WAVES; ++k) {
            ml[k] = *(const float2*)(rml + (k * 16 + row) * 2);
            mm = fmaxf(mm, ml[k].x);
        }
        const float msub = mm == FS_NEG_INF ? 0.f : mm;
        float den = 0.f, wt[WAVES];
#pragma unroll
        for (int k = 0; k < WAVES; ++k) {
            wt[k] = __builtin_amdgcn_exp2f(ml[k].x - msub);
            den += wt[k] * ml[k].y;
        }
#pragma unroll
        for (int u = 0; u < NA; ++u) {
            const int c = (tid & 15) * 4 + u * 64;
            f32x4 o{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < WAVES; ++k) o += *(const f32x4*)(ro + (k * 16 + row) * RROW + c) * wt[k];
            if (a.n_splits == 1) {
                store_row<T>(a, rq, kvh, rho, c, o, den);
            } else {
                const size_t prow = ((size_t)split * a.Hkv + kvh) * a.Rpad + (size_t)a.G * rq.row0 + rho;
                *(f32x4*)(a.part_o + prow * HD + c) = o;
                if (c == 0) *(float2*)(a.part_ml + prow * 2) = make_float2(mm, den);
            }
        }
    }
}

// out = sum_s 2^(m_s - m) O_s / sum_s 2^(m_s - m) l_s.  LANES adjacent lanes share four columns of a row and take splits q, q + LANES, ...,
// then meet pairwise in a fixed order.
template <typename T, int LANES>
__global__ void __launch_bounds__(256) paged_merge_kernel(const PagedArgs a) {
    const int chunks = a.hd / 4, total = a.G * a.rows;
    const int id = (blockIdx.x * 256 + threadIdx.x) / LANES, q = threadIdx.x % LANES;
    const int kvh = blockIdx.y, rho = id / chunks, c = id % chunks * 4;
    if (rho >= total) return;
    const size_t step = (size_t)a.Hkv * a.Rpad, row = (size_t)kvh * a.Rpad + rho;
    float m = FS_NEG_INF, den = 0.f;
    f32x4 o{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = q; s < a.n_splits; s += LANES) {
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
    int rq = 0;
    while (rq + 1 < a.n_req && rho >= a.G * a.req[rq + 1].row0) ++rq;
    store_row<T>(a, a.req[rq], kvh, rho - a.G * a.req[rq].row0, c, o, den);
}

template <typename T, int HD>
hipError_t launch(const PagedArgs& a, int mtw, hipStream_t s) {
    const dim3 grid(a.n_splits, a.Hkv, a.n_req * a.row_blocks), block(WAVES * 64);
    if (mtw == 1) hipLaunchKernelGGL((paged_attn_kernel<T, HD, 1>), grid, block, 0, s, a);
    else if (mtw == 2) hipLaunchKernelGGL((paged_attn_kernel<T, HD, 2>), grid, block, 0, s, a);
    else if constexpr (sizeof(T) == 2) hipLaunchKernelGGL((paged_attn_kernel<T, HD, 4>), grid, block, 0, s, a);
    if (a.n_splits > 1) {
        const int threads = a.G * a.rows * (HD / 4);
        if (a.n_splits >= 4) hipLaunchKernelGGL((paged_merge_kernel<T, 4>), dim3((threads * 4 + 255) / 256, a.Hkv), dim3(256), 0, s, a);
        else hipLaunchKernelGGL((paged_merge_kernel<T, 1>), dim3((threads + 255) / 256, a.Hkv), dim3(256), 0, s, a);
    }
    return hipGetLastError();
}

constexpr int TARGET_WGS = 512;

}  // namespace

int paged_max_splits(int Hkv, int R) { return std::min(64, std::max(1, TARGET_WGS / (Hkv * ((R + 63) / 64)))); }

int paged_plan(int dtype, PagedArgs& a) {
    int R = 0, tiles = 1;
    for (int i = 0; i < a.n_req; ++i) {
        const PagedReq& r = a.req[i];
        R = std::max(R, a.G * r.M);
        tiles = std::max(tiles, (r.n_paged + PAGE_TOK - 1) / PAGE_TOK + (r.l_glo + r.seg_off + r.M - r.n_paged + 63) / 64);
    }
    const int mtw = R <= 16 ? 1 : R <= 32 || dtype == 0 ? 2 : 4;
    a.row_blocks = (R + 16 * mtw - 1) / (16 * mtw);
    const int base = a.n_req * a.Hkv * a.row_blocks;
    int n = std::min(std::min(64, std::max(1, TARGET_WGS / base)), (tiles + WAVES - 1) / WAVES);
    a.tiles_per_split = (tiles + n - 1) / n;
    a.n_splits = (tiles + a.tiles_per_split - 1) / a.tiles_per_split;
    a.Rpad = (a.G * a.rows + 15) / 16 * 16;
    return mtw;
}

hipError_t launch_paged_attention(int dtype, const PagedArgs& a, int mtw, hipStream_t s) {
    if (dtype == 0) return a.hd == 64 ? launch<float, 64>(a, mtw, s) : launch<float, 128>(a, mtw, s);
    return a.hd == 64 ? launch<bf16_t, 64>(a, mtw, s) : launch<bf16_t, 128>(a, mtw, s);
}
