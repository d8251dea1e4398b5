// Attention of one wave over 16-bit or 32-bit key/value rows in memory: what the paged kernel does behind the settled pages and the
// prompt kernel of 32-bit types does everywhere.
//
// A wave owns MTW tiles of 16 query rows.  S^T = K . Q^T and O^T += V^T . P^T keep every quantity of query row l % 16 in lane l (as in
// the tree-attention kernel), so the running maximum and sum are per lane and P stays in registers.  The contraction of S^T runs over
// the columns in the order col(kt, g, e) = 64 (kt / per) + 16 g + EPF (kt % per) + e, per = 64 / KT: a lane's 16 columns of a group
// of 64 are contiguous, which is one 16-byte load for 8-bit codes.
#pragma once
#include "common.hpp"

#define FS_NEG_INF (-__builtin_inff())

template <typename T, int HD, int MTW>
struct RowTiles {
    using E = Elem<T>;
    using frag_t = typename E::frag_t;
    static constexpr int EPF = E::EPF, KT = E::KT, PER = 64 / KT;
    static constexpr int NKT = HD / KT, NHT = HD / 16, NSUB = EPF / 4;
    static constexpr int HS = 32;                       // slots of a half tile, the unit of the loop over rows in memory
    static constexpr int VROW = HD + 16 / (int)sizeof(T);  // padded row of the staged V half
    static constexpr int STAGE = HS * VROW;             // elements of LDS per wave
    static constexpr int NCC = HD / EPF;                // 16-byte chunks of a row
    static constexpr int VCH = HS * NCC / 64;           // chunks of a V half per lane

    // The running maximum is only raised where a score exceeds it by more than this (base 2): any common factor of numerator and
    // denominator is as good, and 8 bits of headroom cost a floating-point sum no precision; most tiles then rescale nothing.
    static constexpr float HEADROOM = 8.f;

    frag_t qf[MTW][NKT];
    f32x4 acc[MTW][NHT];
    float m[MTW], ms[MTW], l[MTW];  // ms: what is subtracted from the scores: m, or 0 while nothing has been seen

    static __device__ __forceinline__ int col(int kt, int g) { return (kt / PER) * 64 + g * 16 + (kt % PER) * EPF; }

    __device__ __forceinline__ void init() {
#pragma unroll
        for (int i = 0; i < MTW; ++i) {
            m[i] = FS_NEG_INF;
            ms[i] = 0.f;
            l[i] = 0.f;
#pragma unroll
            for (int nt = 0; nt < NHT; ++nt) acc[i][nt] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
    __device__ __forceinline__ void load_q(int i, const T* row, bool ok, int g) {
#pragma unroll
        for (int kt = 0; kt < NKT; ++kt) qf[i][kt] = ok ? *(const frag_t*)(row + col(kt, g)) : E::zero();
    }

    // Scores of JN sub-tiles of 16 slots -> probabilities, with the running maximum and sum brought up to date.  vis[i]: bit 16 j + v is
    // set where slot 16 j + 4 g + v counts for row tile i (already shifted by 4 g).  st becomes P (f32).
    template <int JN, bool MASKED>
    __device__ __forceinline__ void softmax(int i, f32x4 (&st)[JN], float scale_log2, unsigned long long vis) {
        float mx = FS_NEG_INF;
#pragma unroll
        for (int j = 0; j < JN; ++j)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                if (MASKED) {
                    const unsigned half = (j * 16 + v) < 32 ? (unsigned)vis : (unsigned)(vis >> 32);
                    st[j][v] = (half & (1u << ((j * 16 + v) & 31))) ? st[j][v] : FS_NEG_INF;
                }
                mx = fmaxf(mx, st[j][v]);
            }
        mx *= scale_log2;  // positive: the maximum commutes with it
        mx = wave_xor_max(wave_xor_max(mx, 16), 32);
        if (__ballot(mx > m[i] + HEADROOM) != 0) {
            const float mnew = fmaxf(m[i], mx);
            ms[i] = mnew == FS_NEG_INF ? 0.f : mnew;
            const float alpha = __builtin_amdgcn_exp2f(m[i] - ms[i]);
            l[i] *= alpha;
#pragma unroll
            for (int nt = 0; nt < NHT; ++nt)
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[i][nt][v] *= alpha;
            m[i] = mnew;
        }
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < JN; ++j)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(st[j][v], scale_log2, -ms[i]));
                st[j][v] = e;
                sum += e;
            }
        l[i] += sum;
    }

    // Operand of the second product: P rounded to the element type (bf16: half a step is 2^-8 of a probability, of the size of the
    // output's own rounding; the sum l is of the unrounded values).
    template <int JN>
    static __device__ __forceinline__ frag_t pack_p(const f32x4 (&p)[JN], int jj) {
        frag_t f;
#pragma unroll
        for (int e = 0; e < EPF; ++e) f[e] = E::from_f(p[jj * NSUB + e / 4][e % 4]);
        return f;
    }

    // 32 slots from rows in memory: slot r of the half at kp / vp + r * stride (elements), rows behind `last` re-read row `last`
    // (they are masked).  vis32[i]: which of the 32 slots row tile i's row sees (MASKED).  vt: the wave's LDS.
    // A masked slot counts for nothing whatever its V row holds: 0 * inf in the matrix product would not, so a half that holds a
    // non-finite value is multiplied slot by slot.
    template <bool MASKED>
    __device__ __forceinline__ void half(const T* kp, const T* vp, long long k_stride, long long v_stride, int last, const unsigned (&vis32)[MTW],
                                         float scale_log2, T* vt, int lane) {
        const int r16 = lane & 15, g = lane >> 4;
        frag_t vr[VCH];
#pragma unroll
        for (int c = 0; c < VCH; ++c) {
            const int ch = lane + 64 * c;
            vr[c] = *(const frag_t*)(vp + (long long)min(ch / NCC, last) * v_stride + (ch % NCC) * EPF);
        }
        f32x4 st[MTW][2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int i = 0; i < MTW; ++i) st[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
            const T* kr = kp + (long long)min(j * 16 + r16, last) * k_stride;
#pragma unroll
            for (int kt = 0; kt < NKT; ++kt) {
                const frag_t kf = *(const frag_t*)(kr + col(kt, g));
#pragma unroll
                for (int i = 0; i < MTW; ++i) st[i][j] = E::mma(kf, qf[i][kt], st[i][j]);
            }
        }
        bool odd = false;
#pragma unroll
        for (int c = 0; c < VCH; ++c) {
            const int ch = lane + 64 * c;
            *(frag_t*)(vt + (ch / NCC) * VROW + (ch % NCC) * EPF) = vr[c];
            if (MASKED) {
                const u32x4 b = __builtin_bit_cast(u32x4, vr[c]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (sizeof(T) == 4) odd |= (b[e] & 0x7f800000u) == 0x7f800000u;
                    else odd |= (((b[e] & 0x7f807f80u) + 0x00800080u) & 0x80008000u) != 0;  // an exponent of all ones in either half
                }
            }
        }
        // the wave's own stores before its own loads of other lanes' data
        __builtin_amdgcn_wave_barrier();
        FS_WAIT_VM_LGKM(63, 0);
        asm volatile("" ::: "memory");
#pragma unroll
        for (int i = 0; i < MTW; ++i) softmax<2, MASKED>(i, st[i], scale_log2, MASKED ? (unsigned long long)(vis32[i] >> (g * 4)) : 0ull);
        if (MASKED && __ballot(odd) != 0) {
#pragma nounroll
            for (int s = 0; s < HS; ++s) {
                const int j = s >> 4, v = s & 3, from = r16 + 16 * ((s >> 2) & 3);
#pragma unroll
                for (int i = 0; i < MTW; ++i) {
                    float p = st[i][0][0];  // value (j, v), by selects: registers have no index
#pragma unroll
                    for (int k = 1; k < 8; ++k) p = k == j * 4 + v ? st[i][k / 4][k % 4] : p;
                    p = __shfl(p, from, FS_WAVE);
                    const bool seen = (vis32[i] >> s) & 1;
#pragma unroll
                    for (int nt = 0; nt < NHT; ++nt) {
                        const typename E::out4_t x = *(const typename E::out4_t*)(vt + s * VROW + nt * 16 + g * 4);
#pragma unroll
                        for (int c = 0; c < 4; ++c)
                            if (seen) acc[i][nt][c] += p * E::to_f(x[c]);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            }
        } else {
#pragma unroll
            for (int jj = 0; jj < 2 / NSUB; ++jj) {
                frag_t pf[MTW];
#pragma unroll
                for (int i = 0; i < MTW; ++i) pf[i] = pack_p<2>(st[i], jj);
#pragma unroll
                for (int nt = 0; nt < NHT; ++nt) {
                    frag_t vf;
                    if constexpr (sizeof(T) == 2) {
                        // transposing load, as in the tree-attention kernel: rows 4 g + r16 / 4 and + 16
                        const T* p0 = vt + (g * 4 + (r16 >> 2)) * VROW + nt * 16 + (r16 & 3) * 4;
                        const s16x4 t0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p0);
                        const s16x4 t1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p0 + 16 * VROW));
                        vf = __builtin_bit_cast(frag_t, __builtin_shufflevector(t0, t1, 0, 1, 2, 3, 4, 5, 6, 7));
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) vf[e] = vt[(jj * 16 + g * 4 + e) * VROW + nt * 16 + r16];
                    }
#pragma unroll
                    for (int i = 0; i < MTW; ++i) acc[i][nt] = E::mma(vf, pf[i], acc[i][nt]);
                }
            }
        }
        // this half's reads of the LDS before the next one's stores
        asm volatile("" ::: "memory");
        __builtin_amdgcn_wave_barrier();
    }
    // the row's sum over the four lanes that share it
    __device__ __forceinline__ float row_sum(int i) const { return wave_xor_add(wave_xor_add(l[i], 16), 32); }
};
