// Pages of 64 tokens in 8 bits: quantising cache rows into them, and the bookkeeping of the sequences that share a pool.
//
// A tile is one (page, layer, K or V, head): 64 rows of hd values as e4m3 codes with one scale 2^e, e the smallest integer with
// max |x| <= 448 * 2^e (at least -117, so that the smallest step, 2^(e - 9), is a normal bf16 number).  A power of two costs a
// floating format no precision and makes both directions exact but for the one rounding to four significant bits.
#include "paged.hpp"

#include <algorithm>

namespace {

// ---- store -------------------------------------------------------------------------------------------------------------------------
// One workgroup per tile: rows -> registers, maximum over the workgroup, codes; K codes leave as they are, V codes through LDS, transposed.
// Bound: the stream, 2 or 4 bytes in and 1 out per element (4 layers x 1500 tokens x 32 heads of 128, bf16: 149 MB in 33.6 us, 4.4 TB/s, the median of 60 traced launches).
template <typename T, int HD>
__global__ void __launch_bounds__(256) paged_store_kernel(const StoreArgs a) {
    using E = Elem<T>;
    using frag_t = typename E::frag_t;
    constexpr int EPF = E::EPF, NCC = HD / EPF, CPT = PAGE_TOK * NCC / 256, ROW = HD + 4;
    __shared__ float red[4];
    __shared__ __align__(16) unsigned char vt[PAGE_TOK * ROW];
    const int tid = threadIdx.x, pg = blockIdx.y, tl = blockIdx.x;  // page of the call, tile of the page: (layer, kv, head)
    int i = 0;
    while (i + 1 < a.n && pg >= a.it[i + 1].page0) ++i;
    const StoreItem& it = a.it[i];
    const PoolDev& p = a.p;
    const int k = pg - it.page0, id = p.table[(size_t)it.seq * p.max_pages + it.first_page + k];
    // only a page that is the sequence's own is written: not one that another sequence reads, not an entry that is no page
    const bool own = (unsigned)id < (unsigned)p.n_pages && p.ref[id] == 1;
    if (tl == 0 && tid == 0 && a.written) a.written[pg] = own;
    if (!own) return;
    const int head = tl % p.Hkv, kv = tl / p.Hkv & 1, layer = tl / p.Hkv >> 1;
    const int n = min(PAGE_TOK, it.n_tokens - k * PAGE_TOK);
    const T* src = (const T*)it.base + layer * it.stride_layer + kv * it.stride_kv + head * it.stride_head + (long long)k * PAGE_TOK * it.stride_tok;

    frag_t x[CPT];
#pragma unroll
    for (int c = 0; c < CPT; ++c) {
        const int ch = tid + c * 256, r = ch / NCC;
        x[c] = r < n ? *(const frag_t*)(src + r * it.stride_tok + (ch % NCC) * EPF) : E::zero();
    }
    float top = 0.f;  // of the finite values
    bool odd = false;
#pragma unroll
    for (int c = 0; c < CPT; ++c)
#pragma unroll
        for (int e = 0; e < EPF; ++e) {
            const float v = fabsf(E::to_f(x[c][e]));
            const bool fine = v < __builtin_inff();
            odd |= !fine;
            top = fine ? fmaxf(top, v) : top;
        }
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) top = wave_xor_max(top, m);
    if ((tid & 63) == 0) red[tid >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    // top = 1.f * 2^(E - 127) and 448 = 1.75 * 2^8: e = E - 135, one more where the fraction is over 0.75
    const unsigned bits = __float_as_uint(top);
    const int e2 = max((int)(bits >> 23) - 135 + ((bits & 0x7fffff) > 0x600000 ? 1 : 0), -117);
    const float up = __uint_as_float((unsigned)(127 - e2) << 23);
    // At the largest scale, 2^120, the codes from 256 on stand for 2^128 and more.  Finite values that round there, 248 * 2^120 and up, take the code
    // below, 240, which is as near as half a step (2^-4 of the value) too.
    if (top >= 0x1.fp127f) {
#pragma unroll
        for (int c = 0; c < CPT; ++c)
#pragma unroll
            for (int e = 0; e < EPF; ++e) {
                const float v = E::to_f(x[c][e]);
                if (fabsf(v) < __builtin_inff()) x[c][e] = E::from_f(fminf(fmaxf(v, -0x1.ep127f), 0x1.ep127f));
            }
    }

    const long long tile = (long long)id * (p.n_layers * 2 * p.Hkv) + tl;
    unsigned char* dst = p.codes + tile * (PAGE_TOK * HD);
    if (tid == 0) p.scales[tile] = __uint_as_float((unsigned)(127 + e2) << 23);
#pragma unroll
    for (int c = 0; c < CPT; ++c) {
        const int ch = tid + c * 256, r = ch / NCC, col = (ch % NCC) * EPF;
        unsigned w[EPF / 4];
#pragma unroll
        for (int q = 0; q < EPF / 4; ++q) {
            const float v0 = E::to_f(x[c][4 * q]) * up, v1 = E::to_f(x[c][4 * q + 1]) * up;
            const float v2 = E::to_f(x[c][4 * q + 2]) * up, v3 = E::to_f(x[c][4 * q + 3]) * up;
            int u = __builtin_amdgcn_cvt_pk_fp8_f32(v0, v1, 0, false);
            w[q] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(v2, v3, u, true);
        }
        if (odd) {  // a value that is not finite becomes the NaN code
#pragma unroll
            for (int e = 0; e < EPF; ++e)
                if (!(fabsf(E::to_f(x[c][e])) < __builtin_inff())) w[e / 4] = (w[e / 4] & ~(0xffu << (8 * (e & 3)))) | (0x7fu << (8 * (e & 3)));
        }
        unsigned char* to = kv ? vt + r * ROW + col : dst + (col >> 6) * (PAGE_TOK * 64) + r * 64 + (col & 63);
#pragma unroll
        for (int q = 0; q < EPF / 4; ++q) *(unsigned*)(to + 4 * q) = w[q];
    }
    if (!kv) return;
    __syncthreads();
#pragma unroll
    for (int c = 0; c < HD * 4 / 256; ++c) {
        const int d = (tid + c * 256) >> 2, g = tid & 3;
        u32x4 o;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const unsigned char* v = vt + (q * 16 + g * 4) * ROW + d;
            o[q] = (unsigned)v[0] | (unsigned)v[ROW] << 8 | (unsigned)v[2 * ROW] << 16 | (unsigned)v[3 * ROW] << 24;
        }
        *(u32x4*)(dst + d * PAGE_TOK + g * 16) = o;
    }
}

// ---- bookkeeping -------------------------------------------------------------------------------------------------------------------
// The reference counts are the whole truth: a page is free where its count is zero, and what is taken is always the lowest free ones.  One workgroup
// decides (about 4 us for up to 4096 pages, most of it latency), a second launch moves the contents.
constexpr int BOOK = 1024;  // threads of the one workgroup that decides
constexpr int W_HEAD = 16;  // work: [0] go-ahead, then two lists of n_pages entries together, then a map of n_pages

static __device__ __forceinline__ int up64(int n) { return (n + PAGE_TOK - 1) / PAGE_TOK; }

// Exclusive prefix sum over the workgroup of one number per thread, and their total.
static __device__ __forceinline__ int block_scan(int v, int* total, int* lds /* [BOOK / 64] */) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    int s = v;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const int t = __shfl_up(s, m, FS_WAVE);
        if (lane >= m) s += t;
    }
    __syncthreads();  // the previous use of lds is over
    if (lane == 63) lds[w] = s;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int i = 0; i < BOOK / 64; ++i) {
        const int t = lds[i];
        before += i < w ? t : 0;
        all += t;
    }
    *total = all;
    return before + s - v;
}

// The `want` lowest free pages into list (fewer if there are not so many); returns how many.
static __device__ int find_free(const PoolDev& p, int want, int32_t* list, int* lds) {
    int found = 0;
    for (int at = 0; at < p.n_pages && found < want; at += BOOK * 4) {
        int idx = at + threadIdx.x * 4, f[4], n = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            f[e] = idx + e < p.n_pages && p.ref[idx + e] == 0;
            n += f[e];
        }
        int total, k = found + block_scan(n, &total, lds);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (f[e] && k < want) list[k++] = idx + e;
        found += total;
    }
    return min(found, want);
}

// l.a sequences, l.b their new lengths in tokens.
__global__ void __launch_bounds__(BOOK) page_grow_kernel(const PoolDev p, const SeqLists l, int32_t* status) {
    __shared__ int lds[BOOK / 64], before[SEQ_LIST + 1], refused;
    __shared__ unsigned long long asked;  // 256 sequences of 2^24 pages each are 2^32
    const int tid = threadIdx.x;
    if (tid == 0) {
        refused = 0;
        asked = 0;
    }
    __syncthreads();
    int need = 0;
    if (tid < l.n) {
        const int len = p.length[l.a[tid]], to = l.b[tid];
        if (len < 0 || to < len) refused = 1;
        need = max(up64(to) - up64(max(len, 0)), 0);
        atomicAdd(&asked, (unsigned long long)need);  // whole numbers: no order matters
    }
    __syncthreads();
    const bool fits = asked <= (unsigned long long)p.n_pages;
    int total;
    const int mine = block_scan(fits ? need : 0, &total, lds);
    if (tid < l.n) before[tid] = mine;
    if (tid == 0) before[l.n] = total;
    __syncthreads();
    int32_t* list = p.work + W_HEAD;
    if (refused || !fits || find_free(p, total, list, lds) < total) {
        if (tid == 0) *status = refused ? -2 : -1;
        return;
    }
    __syncthreads();  // the list is read by other threads
    for (int k = tid; k < total; k += BOOK) {
        int lo = 0, hi = l.n - 1;  // the sequence that takes the k-th page
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (before[mid] <= k) lo = mid;
            else hi = mid - 1;
        }
        const int sq = l.a[lo], id = list[k];
        p.table[(size_t)sq * p.max_pages + up64(p.length[sq]) + k - before[lo]] = id;
        p.ref[id] = 1;
    }
    __syncthreads();  // every length is read before it changes
    if (tid < l.n) p.length[l.a[tid]] = l.b[tid];
    if (tid == 0) *status = total;
}

// l.a sources, l.b destinations: takes a page for every source whose last page is partial.
__global__ void __launch_bounds__(BOOK) page_fork_plan_kernel(const PoolDev p, const SeqLists l, int32_t* status) {
    __shared__ int lds[BOOK / 64], refused;
    const int tid = threadIdx.x;
    if (tid == 0) refused = 0;
    __syncthreads();
    int len = 0;
    if (tid < l.n) {
        len = p.length[l.a[tid]];
        if (p.length[l.b[tid]] != 0 || len < 0 || len > p.max_pages * PAGE_TOK) refused = 1;
    }
    const int part = tid < l.n && len % PAGE_TOK != 0;
    int total;
    const int mine = block_scan(part, &total, lds);
    int32_t* list = p.work + W_HEAD;  // [0, n): the new page of each pair or -1; behind it the free pages found
    int32_t* found = list + l.n;
    if (refused || find_free(p, total, found, lds) < total) {
        if (tid == 0) {
            *status = refused ? -2 : -1;
            p.work[0] = 0;
        }
        return;
    }
    __syncthreads();
    if (tid < l.n) {
        const int id = part ? found[mine] : -1;
        list[tid] = id;
        if (part) p.ref[id] = 1;
        p.length[l.b[tid]] = len;
    }
    if (tid == 0) {
        *status = total;
        p.work[0] = 1;
    }
}

// Bytes of a page (a fork's 16 pages of 2 MB take 13.1 us, a compaction's 117 MB 43.3, medians, reading and writing at 5 TB/s and more): 16-byte pieces [x * 256 + tid, ...) of its codes, then its scales.
static __device__ __forceinline__ void copy_page(const PoolDev& to, int dst, const PoolDev& from, int src, int x, int nx) {
    const int tiles = to.n_layers * 2 * to.Hkv;
    const long long pieces = (long long)tiles * (PAGE_TOK * to.hd / 16);
    const u32x4* s = (const u32x4*)from.codes + src * pieces;
    u32x4* d = (u32x4*)to.codes + dst * pieces;
    // four loads in flight per thread
    for (long long i = (long long)x * 1024 + threadIdx.x; i < pieces; i += (long long)nx * 1024) {
        u32x4 v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (i + e * 256 < pieces) v[e] = __builtin_nontemporal_load(s + i + e * 256);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (i + e * 256 < pieces) __builtin_nontemporal_store(v[e], d + i + e * 256);
    }
    if (x == 0)
        for (int i = threadIdx.x; i < tiles; i += 256) to.scales[(long long)dst * tiles + i] = from.scales[(long long)src * tiles + i];
}

__global__ void __launch_bounds__(256) page_fork_kernel(const PoolDev p, const SeqLists l) {
    if (p.work[0] == 0) return;
    const int i = blockIdx.y, src = l.a[i], dst = l.b[i], len = p.length[src], full = len / PAGE_TOK, id = p.work[W_HEAD + i];
    const int32_t* from = p.table + (size_t)src * p.max_pages;
    if (blockIdx.x == 0) {
        int32_t* to = p.table + (size_t)dst * p.max_pages;
        for (int k = threadIdx.x; k < p.max_pages; k += 256) {
            int e = -1;
            if (k < full) {
                e = from[k];
                if ((unsigned)e < (unsigned)p.n_pages) atomicAdd(&p.ref[e], 1);  // whole numbers: no order matters
            } else if (k == full) {
                e = id;
            }
            to[k] = e;
        }
    }
    if (id >= 0) {
        const int old = from[full];
        if ((unsigned)old < (unsigned)p.n_pages) copy_page(p, id, p, old, blockIdx.x, gridDim.x);
    }
}

__global__ void __launch_bounds__(256) page_free_kernel(const PoolDev p, const SeqLists l) {
    const int sq = l.a[blockIdx.x], n = min(up64(max(p.length[sq], 0)), p.max_pages);
    int32_t* row = p.table + (size_t)sq * p.max_pages;
    for (int k = threadIdx.x; k < n; k += 256) {
        const int id = row[k];
        if ((unsigned)id < (unsigned)p.n_pages) atomicSub(&p.ref[id], 1);
        row[k] = -1;
    }
    __syncthreads();  // every thread has read the length
    if (threadIdx.x == 0) p.length[sq] = 0;
}

// The k-th live page behind the first `live` pages moves to the k-th free page among them: sources and destinations never meet.
__global__ void __launch_bounds__(BOOK) page_compact_plan_kernel(const PoolDev p, int32_t* status) {
    __shared__ int lds[BOOK / 64];
    const int tid = threadIdx.x, n = p.n_pages;
    int mine = 0, live;
    for (int i = tid; i < n; i += BOOK) mine += p.ref[i] > 0;
    block_scan(mine, &live, lds);
    int32_t *src = p.work + W_HEAD, *dst = src + (n + 1) / 2, *map = src + n + 1;
    int ns = 0, nd = 0;
    for (int at = 0; at < n; at += BOOK) {
        const int i = at + tid;
        const bool used = i < n && p.ref[i] > 0;
        const int s = used && i >= live, d = i < live && !used;  // (i < live implies i < n)
        int t, k = block_scan(s | d << 16, &t, lds);
        if (s) src[ns + (k & 0xffff)] = i;
        if (d) dst[nd + (k >> 16)] = i;
        if (i < n) map[i] = i;
        ns += t & 0xffff;
        nd += t >> 16;
    }
    __syncthreads();
    // (as many live pages behind the line as free ones before it)
    for (int k = tid; k < ns; k += BOOK) {
        const int s = src[k], d = dst[k];
        map[s] = d;
        p.ref[d] = p.ref[s];
        p.ref[s] = 0;
    }
    if (tid == 0) {
        p.work[0] = ns;
        *status = ns;
    }
}

__global__ void __launch_bounds__(256) page_compact_kernel(const PoolDev p, int per_page) {
    const int moves = p.work[0];
    if (moves == 0) return;
    const int32_t *src = p.work + W_HEAD, *dst = src + (p.n_pages + 1) / 2, *map = src + p.n_pages + 1;
    // tables: a row per workgroup in turn
    for (int sq = blockIdx.x; sq < p.n_seqs; sq += gridDim.x) {
        int32_t* row = p.table + (size_t)sq * p.max_pages;
        for (int k = threadIdx.x; k < p.max_pages; k += 256) {
            const int id = row[k];
            if ((unsigned)id < (unsigned)p.n_pages) row[k] = map[id];
        }
    }
    for (int j = blockIdx.x; j < moves * per_page; j += gridDim.x) copy_page(p, dst[j / per_page], p, src[j / per_page], j % per_page, per_page);
}

__global__ void __launch_bounds__(256) page_copy_kernel(const PoolDev to, const PoolDev from, const SeqLists l) {
    copy_page(to, l.b[blockIdx.y], from, l.a[blockIdx.y], blockIdx.x, gridDim.x);
}

// Workgroups per page: 16 KiB each, fewer where there are many pages to move.
int page_groups(const PoolDev& p, int pages) {
    const long long pieces = (long long)p.n_layers * 2 * p.Hkv * (PAGE_TOK * p.hd / 16);
    return (int)std::max<long long>(1, std::min<long long>((pieces + 1023) / 1024, std::max(1, 4096 / std::max(1, pages))));
}

}  // namespace

hipError_t launch_paged_store(int dtype, const StoreArgs& a, int pages, hipStream_t s) {
    const dim3 grid(a.p.n_layers * 2 * a.p.Hkv, pages);
    if (dtype == 0) {
        if (a.p.hd == 64) hipLaunchKernelGGL((paged_store_kernel<float, 64>), grid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL((paged_store_kernel<float, 128>), grid, dim3(256), 0, s, a);
    } else {
        if (a.p.hd == 64) hipLaunchKernelGGL((paged_store_kernel<bf16_t, 64>), grid, dim3(256), 0, s, a);
        else hipLaunchKernelGGL((paged_store_kernel<bf16_t, 128>), grid, dim3(256), 0, s, a);
    }
    return hipGetLastError();
}

hipError_t launch_page_grow(const PoolDev& p, const SeqLists& l, int32_t* status, hipStream_t s) {
    hipLaunchKernelGGL(page_grow_kernel, dim3(1), dim3(BOOK), 0, s, p, l, status);
    return hipGetLastError();
}

hipError_t launch_page_fork(const PoolDev& p, const SeqLists& l, int32_t* status, hipStream_t s) {
    hipLaunchKernelGGL(page_fork_plan_kernel, dim3(1), dim3(BOOK), 0, s, p, l, status);
    hipLaunchKernelGGL(page_fork_kernel, dim3(page_groups(p, l.n), l.n), dim3(256), 0, s, p, l);
    return hipGetLastError();
}

hipError_t launch_page_free(const PoolDev& p, const SeqLists& l, hipStream_t s) {
    hipLaunchKernelGGL(page_free_kernel, dim3(l.n), dim3(256), 0, s, p, l);
    return hipGetLastError();
}

hipError_t launch_page_compact(const PoolDev& p, int32_t* status, hipStream_t s) {
    hipLaunchKernelGGL(page_compact_plan_kernel, dim3(1), dim3(BOOK), 0, s, p, status);
    const int per = page_groups(p, 64);
    hipLaunchKernelGGL(page_compact_kernel, dim3(2048), dim3(256), 0, s, p, per);
    return hipGetLastError();
}

hipError_t launch_page_copy(const PoolDev& dst, const PoolDev& src, const SeqLists& l, hipStream_t s) {
    hipLaunchKernelGGL(page_copy_kernel, dim3(page_groups(dst, l.n), l.n), dim3(256), 0, s, dst, src, l);
    return hipGetLastError();
}
